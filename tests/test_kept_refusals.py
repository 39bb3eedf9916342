"""What the entry points of the 8-bit checkpoints refuse, before any launch (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kept_oracle
from paper_2605_05838_amd import binding


def test_the_oracle_at_values_worked_out_by_hand():
    x = np.zeros((1, 64))
    x[0, :5] = [1.0, 1.0 / 64, 1.5 / 64, -2.5 / 64, 127.6 / 64]      # largest 1.99: step 1/64
    x[0, 32:35] = [3.0, 100.0, -0.7]                                  # largest 100: step 1
    y = kept_oracle.values(x)[0]
    assert y[:5].tolist() == [1.0, 1.0 / 64, 2.0 / 64, -2.0 / 64, 127.0 / 64] and y[32:35].tolist() == [3.0, 100.0, -1.0]


def shape(**kw):
    s = dict(B=2, T=5, H=3, dk=64, dv=64, C=64, dtype=0, scale=1.0)
    s.update(kw)
    return binding.MdnShape(**s)


P = ctypes.c_void_p(4096)
KEPT = (binding.MdnKept * 3)(*[binding.MdnKept(4096, 4096)] * 3)
HOLES = [(binding.MdnKept * 3)(*[binding.MdnKept(*p)] * 3) for p in ((None, 4096), (4096, None))] + [None]


def calls(lib, s, kept=KEPT, p=P, ws=P, n=1 << 40):
    f, b = ctypes.c_float(1e-6), ctypes.byref
    return [lib.mdn_keep(b(s), p, kept, None), lib.mdn_kept_values(b(s), kept, p, None),
            lib.mdn_frontend_fwd_keep(b(s), p, p, p, p, f, p, p, p, kept, None), lib.mdn_frontend_fwd_kept(b(s), kept, p, f, p, p, p, None),
            lib.mdn_frontend_bwd_kept(b(s), kept, p, f, p, p, p, p, p, p, p, ws, n, None),
            lib.mdn_epilogue_fwd_keep(b(s), p, p, p, f, p, kept, None),
            lib.mdn_epilogue_bwd_kept(b(s), kept, p, f, p, p, p, p, ws, n, None)]


@pytest.mark.parametrize("bad,code", [(dict(T=0), -2), (dict(dk=32, dv=32), -2), (dict(dk=64, dv=128), -2), (dict(H=5000), -2), (dict(dtype=3), -3)])
def test_shapes(bad, code):
    lib, n = binding.load_library(), ctypes.c_size_t(0)
    assert set(calls(lib, shape(**bad))) == {code}
    assert lib.mdn_kept_workspace_bytes(ctypes.byref(shape(**bad)), ctypes.byref(n)) == code


def test_pointers_and_workspace():
    lib, n = binding.load_library(), ctypes.c_size_t(0)
    for kept in HOLES:
        assert set(calls(lib, shape(), kept=kept)) == {-1}
    assert set(calls(lib, shape(), p=None)) == {-1}
    assert calls(lib, shape(), ws=None)[4::2] == [-1, -1]
    assert calls(lib, shape(), ws=ctypes.c_void_p(4098))[4::2] == [-5, -5]
    assert calls(lib, shape(), n=8)[4::2] == [-4, -4]
    assert lib.mdn_kept_workspace_bytes(ctypes.byref(shape()), ctypes.byref(n)) == 0 and n.value > 0
    assert lib.mdn_kept_workspace_bytes(ctypes.byref(shape()), None) == -1


def test_tensors():
    x = torch.zeros(2, 5, 3, 64)
    kept = (torch.zeros(2, 5, 3, 64, dtype=torch.int8), torch.zeros(2, 5, 3, 2, dtype=torch.uint8))
    d, w = torch.zeros(3), torch.zeros(64)
    refused = [lambda: binding.mdn_keep(x), lambda: binding.mdn_keep(x[0]), lambda: binding.mdn_keep(x[..., :32]), lambda: binding.mdn_keep(x.half()),
               lambda: binding.mdn_keep(x.transpose(1, 2)), lambda: binding.mdn_kept_values(kept, torch.float32),
               lambda: binding.mdn_kept_values(kept, torch.float16), lambda: binding.mdn_kept_values(kept[0], torch.float32),
               lambda: binding.mdn_kept_values((kept[0], kept[1][..., :1]), torch.float32),
               lambda: binding.mdn_kept_values((kept[1], kept[0]), torch.float32),
               lambda: binding.mdn_frontend_fwd_keep(x, x, x, d), lambda: binding.mdn_frontend_fwd_keep(x, x, x, w),
               lambda: binding.mdn_frontend_fwd_keep(x, x, torch.zeros(2, 5, 3, 128), d),
               lambda: binding.mdn_frontend_fwd_kept(kept, kept, (kept[0][:1], kept[1][:1]), d, torch.float32),
               lambda: binding.mdn_frontend_fwd_kept(kept, kept, kept, d, torch.float32),
               lambda: binding.mdn_frontend_bwd_kept(kept, kept, kept, d, x, x, x.bfloat16()),
               lambda: binding.mdn_frontend_bwd_kept(kept, kept, kept, d, x, x, x),
               lambda: binding.mdn_epilogue_fwd_keep(x, x, w), lambda: binding.mdn_epilogue_fwd_keep(x, x[:1], w),
               lambda: binding.mdn_epilogue_bwd_kept(kept, kept, d, x), lambda: binding.mdn_epilogue_bwd_kept(kept, kept, w, x)]
    for call in refused:
        with pytest.raises(binding.MdnError):
            call()
