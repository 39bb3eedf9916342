"""What the gated delta rule's entry points refuse, before any launch (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2605_05838_amd import binding


def shape(**kw):
    s = dict(B=2, T=128, H=4, Hk=2, dk=128, dv=128, dtype=0, scale=0.1)
    s.update(kw)
    return binding.MdnGdrShape(**s)


def bytes_rc(s, cu=None, which=0):
    n = ctypes.c_size_t(0)
    arr = None if cu is None else (ctypes.c_int32 * len(cu))(*cu)
    return binding.load_library().mdn_gdr_bytes(ctypes.byref(s), arr, 0 if cu is None else len(cu) - 1, which, ctypes.byref(n)), n.value


@pytest.mark.parametrize("bad,code", [(dict(T=0), -2), (dict(B=0), -2), (dict(H=3), -2), (dict(Hk=0), -2), (dict(H=8192, Hk=8192), -2),
                                      (dict(dk=96), -2), (dict(dv=256), -2), (dict(dtype=2), -3), (dict(B=1 << 20, H=32, Hk=32), -2),
                                      (dict(B=1 << 12, T=1 << 18), -2)])
def test_shapes(bad, code):
    for which in range(4):
        assert bytes_rc(shape(**bad), which=which)[0] == code
    assert binding.load_library().mdn_gdr_recurrent_step(ctypes.byref(shape(**bad)), *[ctypes.c_void_p(4096)] * 7, None) == code


def test_sizes_follow_the_shape():
    blocks = 2 * 2 * 4
    assert bytes_rc(shape(), which=2) == (0, blocks * 128 * 128 * 2)
    assert bytes_rc(shape(T=65), which=2) == (0, blocks * 128 * 128 * 2)
    assert bytes_rc(shape(dtype=1), which=2) == (0, blocks * 128 * 128 * 4)
    assert bytes_rc(shape(), which=3) == (0, blocks * (1024 + 2 * 6144))
    assert bytes_rc(shape(), which=1)[1] > 2 * blocks * 128 * 128 * 2
    assert bytes_rc(shape(), which=4)[0] == -2
    assert binding.gdr_bytes(shape(B=1, T=70), binding.MDN_GDR_STATES, [0, 1, 70]) == 3 * 4 * 128 * 128 * 2
    assert binding.load_library().mdn_gdr_bytes(ctypes.byref(shape()), None, 0, 0, None) == -1


@pytest.mark.parametrize("cu", [[0, 100], [0, 64, 64, 128], [1, 128], [0, 130, 128], [0, -5, 128]])
def test_offsets(cu):
    assert bytes_rc(shape(B=1), cu)[0] == -2
    assert bytes_rc(shape(B=2), [0, 128])[0] == -2
    with pytest.raises(binding.MdnError):
        x = tensors(B=1, T=128)
        binding.mdn_gdr_chunk_fwd(*x, cu_seqlens=cu)


def test_pointers():
    lib, s, good, bad = binding.load_library(), shape(), ctypes.c_void_p(4096), ctypes.c_void_p(4104)
    fwd = [good] * 12
    call = lambda args, n=1 << 40: lib.mdn_gdr_chunk_fwd(ctypes.byref(s), None, 0, *args, n, None)
    for i in (0, 1, 2, 3, 4, 6, 11):
        assert call(fwd[:i] + [None] + fwd[i + 1:]) == -1
    for i in range(12):
        assert call(fwd[:i] + [bad] + fwd[i + 1:]) == -5
    assert call(fwd, 1024) == -4
    assert lib.mdn_gdr_chunk_fwd(ctypes.byref(s), None, 3, *fwd, 1 << 40, None) == -1
    bwd = [good] * 17
    call = lambda args, n=1 << 40: lib.mdn_gdr_chunk_bwd(ctypes.byref(s), None, 0, *args, n, None)
    for i in (0, 1, 2, 3, 5, 8, 10, 11, 12, 13, 14, 16):
        assert call(bwd[:i] + [None] + bwd[i + 1:]) == -1
    for i in range(17):
        assert call(bwd[:i] + [bad] + bwd[i + 1:]) == -5
    assert call(bwd, 1024) == -4


def tensors(B=2, T=10, H=4, Hk=2, dk=64, dv=128, dt=torch.float32):
    z = torch.zeros
    return [z(B, T, Hk, dk, dtype=dt), z(B, T, Hk, dk, dtype=dt), z(B, T, H, dv, dtype=dt), z(B, T, H), z(B, T, H)]


@pytest.mark.parametrize("change", [lambda x: x.__setitem__(1, x[1][:, :9]), lambda x: x.__setitem__(2, x[2].bfloat16()),
                                    lambda x: x.__setitem__(2, torch.zeros(2, 10, 3, 128)), lambda x: x.__setitem__(3, x[3].double()),
                                    lambda x: x.__setitem__(4, x[4].transpose(1, 2)), lambda x: x.__setitem__(0, x[0][0]),
                                    lambda x: x.__setitem__(0, x[0].half()), lambda x: None])
def test_tensors(change):
    """A wrong shape, type, layout, head count; and, last, tensors that are not on the GPU."""
    x = tensors()
    change(x)
    q, k, v, g, beta = x
    with pytest.raises(binding.MdnError):
        binding.mdn_gdr_chunk_fwd(q, k, v, g, beta)
    with pytest.raises(binding.MdnError):
        binding.mdn_gdr_chunk_bwd(q, k, g, beta, v, v)
    with pytest.raises(binding.MdnError):
        binding.mdn_gdr_recurrent_step(q, k, v, g, beta, torch.zeros(2, 4, 64, 128))


def test_states_and_buffers_of_another_size():
    q, k, v, g, beta = tensors()
    with pytest.raises(binding.MdnError, match="S0"):
        binding.mdn_gdr_chunk_fwd(q, k, v, g, beta, S0=torch.zeros(2, 4, 128, 64))
    with pytest.raises(binding.MdnError, match="dS_final"):
        binding.mdn_gdr_chunk_bwd(q, k, g, beta, v, v, dS_final=torch.zeros(1, 4, 64, 128))
    with pytest.raises(binding.MdnError, match="states"):
        binding.mdn_gdr_chunk_bwd(q, k, g, beta, v, v, states=torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(binding.MdnError, match="workspace"):
        binding.mdn_gdr_chunk_fwd(q, k, v, g, beta, workspace=torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(binding.MdnError, match="dO"):
        binding.mdn_gdr_chunk_bwd(q, k, g, beta, v, v[:, :5])
    with pytest.raises(binding.MdnError, match="S is required"):
        binding.mdn_gdr_recurrent_step(q, k, v, g, beta, None)
