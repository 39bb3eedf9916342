"""The gated delta rule's dg and dbeta in 32 bits where the storage type has 16."""
import ctypes
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_2605_05838_amd import binding


def test_the_flag_changes_no_size_and_nothing_else_is_taken():
    lib, n = binding.load_library(), ctypes.c_size_t(0)
    size = lambda dtype, which: (lib.mdn_gdr_bytes(ctypes.byref(binding.MdnGdrShape(2, 128, 4, 2, 128, 64, dtype, 0.1)), None, 0, which, ctypes.byref(n)), n.value)
    for dtype in (0, 1):
        for which in range(4):
            assert size(dtype | binding.MDN_GDR_F32_GATE_GRADS, which) == size(dtype, which) and size(dtype, which)[0] == 0
    for dtype in (2, 3, 8, 17 + 1, 32, 33, -1, -16):
        assert size(dtype, 0)[0] == -3, dtype


def test_refusals():
    z = torch.zeros
    x = lambda dt: (z(1, 9, 2, 64, dtype=dt), z(1, 9, 2, 64, dtype=dt), z(1, 9, 2), z(1, 9, 2), z(1, 9, 2, 64, dtype=dt), z(1, 9, 2, 64, dtype=dt))
    for dt, gate in ((torch.bfloat16, torch.float16), (torch.bfloat16, "float32"), (torch.float32, torch.bfloat16)):
        with pytest.raises(binding.MdnError, match="gate_dtype"):
            binding.mdn_gdr_chunk_bwd(*x(dt), gate_dtype=gate)
    with pytest.raises(binding.MdnError, match="dg"):
        binding.mdn_gdr_chunk_bwd(*x(torch.bfloat16), gate_dtype=torch.float32, out={"dg": z(1, 9, 2, dtype=torch.bfloat16)})


@pytest.mark.gpu
@pytest.mark.parametrize("cu", [None, [0, 1, 70, 300]])
@pytest.mark.parametrize("H,Hk,dk,dv", [(4, 4, 64, 64), (6, 2, 128, 64), (2, 1, 64, 128), (4, 2, 128, 128)])
def test_they_are_what_the_16_bits_are_rounded_from(cu, H, Hk, dk, dv):
    from gdr_util import check, inputs, oracle
    seqs = len(cu) - 1 if cu else 1
    x = inputs("bf16", T=300, H=H, Hk=Hk, dk=dk, dv=dv, seqs=seqs, seed=2)
    f = binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S0=x["S0"], cu_seqlens=cu, save_e=True)
    call = lambda **kw: binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], x["dO"], S0=x["S0"], dS_final=x["dS"], cu_seqlens=cu,
                                                  want_dS0=True, **kw)
    a, b = call(), call(gate_dtype=torch.float32)
    for n in ("dg", "dbeta"):
        assert a[n].dtype == torch.bfloat16 and b[n].dtype == torch.float32 and torch.equal(b[n].bfloat16(), a[n]) and not torch.equal(b[n], a[n].float())
    assert all(torch.equal(a[n], b[n]) for n in ("dq", "dk", "dv", "dS0"))
    check({n: b[n] for n in ("dg", "dbeta")}, {n: w for n, w in oracle(x, cu=cu).items() if n in ("dg", "dbeta")}, "bf16")
    assert torch.equal(call(gate_dtype=torch.float32, out=b)["dg"].bfloat16(), a["dg"])


@pytest.mark.gpu
def test_32_bit_storage_has_them_anyway():
    from gdr_util import inputs
    x = inputs("f32", T=70, seed=3)
    e = binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], save_e=True)["e"]
    a, b = (binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], e, x["dO"], gate_dtype=t) for t in (None, torch.float32))
    assert torch.equal(a["dg"], b["dg"]) and torch.equal(a["dbeta"], b["dbeta"])
