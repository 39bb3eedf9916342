"""Gated delta rule: how far a value reaches.  What is not finite stays in its sequence and, in the forward, behind its chunk's first token; tensors
of more than 2^32 bytes are addressed to their ends."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import inputs, run
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("token", [199, 134, 150]) # the last of its sequence, the first of its second chunk, inside it
@pytest.mark.parametrize("name", ["q", "k", "v", "beta", "dO"])
def test_what_is_not_finite_stays_where_it_may_be(dtype, value, token, name):
    cu = [0, 70, 200, 330]
    x = inputs(dtype, T=330, H=4, Hk=2, dk=64, dv=128, seqs=3, seed=4)
    good = run(x, cu=cu)
    x[name][0, token] = value
    bad = run(x, cu=cu)
    assert not all(torch.isfinite(t).all() for t in bad.values())
    for n in ("o", "e", "dq", "dk", "dv", "dg", "dbeta"):
        assert torch.equal(bad[n][:, :70], good[n][:, :70]) and torch.equal(bad[n][:, 200:], good[n][:, 200:]), n
    for n in ("o", "e"):
        assert torch.equal(bad[n][:, :134], good[n][:, :134]), n
    for n in ("S", "dS0"):
        assert torch.equal(bad[n][[0, 2]], good[n][[0, 2]]), n


def test_tensors_of_more_than_four_gigabytes():
    """v, o, e, dv, dO of 4.5 GB, states of 9 GB: the first and the last heads are bit for bit those of a call of their own."""
    T, H, Hk, d = 1100003, 16, 8, 128
    r = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=r, device="cuda", dtype=torch.bfloat16)
    x = dict(q=n(1, T, Hk, d), k=n(1, T, Hk, d), v=n(1, T, H, d), g=-0.1 * torch.rand(1, T, H, generator=r, device="cuda"),
             beta=torch.rand(1, T, H, generator=r, device="cuda"))
    for m in "qk":
        x[m] /= x[m].norm(dim=-1, keepdim=True)
    dO = n(1, T, H, d)

    def step(x, dO):
        f = binding.mdn_gdr_chunk_fwd(*x.values(), save_e=True, save_states=True)
        b = binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], dO, states=f["states"])
        return {m: f[m] for m in "oeS"} | {m: b[m] for m in ("dq", "dk", "dv", "dg", "dbeta")}
    got = step(x, dO)
    assert x["v"].nbytes > 1 << 32
    for key in (0, Hk - 1):
        heads = slice(2 * key, 2 * key + 2)
        part = {m: (t[:, :, key:key + 1] if m in "qk" else t[:, :, heads]).contiguous() for m, t in x.items()}
        want = step(part, dO[:, :, heads].contiguous())
        for m, t in got.items():
            t = t[:, heads] if m == "S" else t[:, :, key:key + 1] if m in ("dq", "dk") else t[:, :, heads]
            assert torch.equal(t, want[m]), (m, key)
        assert torch.isfinite(got["o"][:, -1]).all()
