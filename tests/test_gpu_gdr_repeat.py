"""Gated delta rule: repeated calls agree bit for bit, whichever waves arrive first."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import inputs
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("B,T,H,Hk,dk,dv", [(1, 777, 16, 16, 128, 128), (4, 2048, 16, 16, 128, 128), (4, 2048, 16, 4, 64, 64), (2, 1500, 8, 2, 64, 128),
                                            (3, 1500, 16, 16, 128, 64)])
def test_repeated_calls(dtype, states, B, T, H, Hk, dk, dv):
    x = inputs(dtype, B=B, T=T, H=H, Hk=Hk, dk=dk, dv=dv, seed=T + dk)
    S0, dS = (x["S0"], x["dS"]) if states else (None, None)

    def call():
        f = binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S0=S0, save_e=True, save_states=True, output_final_state=states)
        b = binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], x["dO"], S0=S0, states=f["states"], dS_final=dS, want_dS0=states)
        r = binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], x["dO"], S0=S0, dS_final=dS)
        return [f[n] for n in ("o", "e", "states", "S")] + [b[n] for n in ("dq", "dk", "dv", "dg", "dbeta", "dS0")] + [r[n] for n in ("dq", "dv", "dg")]
    want = call()
    for i in range(24):
        got = call()
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(got, want)), i
