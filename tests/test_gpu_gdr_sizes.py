"""Gated delta rule where a launch changes form by the size of its tensors: steps on states past the last-level cache, and state
reconstructions that bring later chunks' operands into the L2.  Bit for bit what calls on parts of the same tensors give, which take the
other form, and some of it against the fp64 oracle."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import DT
from gpu_util import host
from oracle import gdr_oracle
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu


def tensors(dtype, B, T, H, Hk, dk, dv, seed):
    r = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=r, device="cuda")
    unit = lambda *s: torch.nn.functional.normalize(n(*s), dim=-1).to(DT[dtype])
    return dict(q=unit(B, T, Hk, dk), k=unit(B, T, Hk, dk), v=n(B, T, H, dv).to(DT[dtype]), g=-0.1 * torch.nn.functional.softplus(n(B, T, H)),
                beta=torch.sigmoid(n(B, T, H))), n


# states of 352 MiB and more: 5 632 pairs of 128 x 128, 11 264 of 64 x 128
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,Hk,dk,dv", [(354, 1, 16, 8, 128, 128), (354, 3, 16, 16, 128, 128), (706, 2, 16, 4, 64, 128)])
def test_step_on_states_past_the_last_level_cache(dtype, B, T, H, Hk, dk, dv):
    x, n = tensors(dtype, B, T, H, Hk, dk, dv, seed=B + T)
    S0 = 0.3 * n(B, H, dk, dv)
    S = S0.clone()
    assert S.nbytes > 352 << 20
    o = binding.mdn_gdr_recurrent_step(*x.values(), S)
    for rows in (slice(0, B // 2), slice(B // 2, B)):
        part = S0[rows].clone()
        assert part.nbytes < 352 << 20
        po = binding.mdn_gdr_recurrent_step(*[t[rows].contiguous() for t in x.values()], part)
        assert torch.equal(S[rows], part) and torch.equal(o[rows], po)
    some = [0, B // 2, B - 1]
    want = gdr_oracle.forward(*[host(t[some]) for t in x.values()], S0=host(S0[some]), scale=dk ** -0.5)
    err = lambda a, b: np.linalg.norm(host(a) - b) / np.linalg.norm(b)
    # fp32 throughout: sums of 128 terms, T of them one after the other; o is rounded once more
    assert err(S[some], want["S"]) < 2e-6 and err(o[some], want["o"]) < (3e-6 if dtype == "f32" else 2.0 ** -8)


def backward(x, e, dO, **kw):
    return binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], e, dO, **kw)


def forward(x, **kw):
    return binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], save_e=True, output_final_state=False, **kw)


@pytest.mark.parametrize("cu", [None, [0, 9001, 9002, 25003]])
def test_reconstruction_few_heads(cu):
    """16 columns a workgroup: 16 value heads on 8, and two value heads by themselves."""
    x, n = tensors("bf16", 1, 25003, 16, 8, 128, 128, seed=1)
    dO = n(1, 25003, 16, 128).bfloat16()
    e = forward(x, cu_seqlens=cu)["e"]
    got = backward(x, e, dO, cu_seqlens=cu)
    for h in range(0, 16, 6):
        part = {m: (t[:, :, h // 2:h // 2 + 1] if m in "qk" else t[:, :, h:h + 2]).contiguous() for m, t in x.items()}
        want = backward(part, *[t[:, :, h:h + 2].contiguous() for t in (e, dO)], cu_seqlens=cu)
        for m in ("dv", "dg", "dbeta"):
            assert torch.equal(got[m][:, :, h:h + 2], want[m]), (h, m)
        for m in ("dq", "dk"):
            assert torch.equal(got[m][:, :, h // 2:h // 2 + 1], want[m]), (h, m)


def test_reconstruction_many_heads():
    """32 columns a workgroup: two sequences of 34 heads, and each by itself."""
    x, n = tensors("bf16", 2, 6394, 34, 34, 128, 128, seed=2) # (an even number: gates of 16-byte alignment in either sequence)
    dO = n(2, 6394, 34, 128).bfloat16()
    e = forward(x)["e"]
    got = backward(x, e, dO)
    for b in range(2):
        want = backward({m: t[b:b + 1] for m, t in x.items()}, e[b:b + 1], dO[b:b + 1])
        for m in ("dq", "dk", "dv", "dg", "dbeta"):
            assert torch.equal(got[m][b:b + 1], want[m]), (b, m)
