"""Gradients of strong decays: every term of dg_t carries e^{g_t}, so that it is as exact behind a strong decay as behind a weak one, and 0 where
the decay is."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import inputs, run
from gpu_util import host
from oracle import gdr_oracle

pytestmark = pytest.mark.gpu
# one to a head: first and last of a chunk, around the borders of 16 tokens, in each quarter of a chunk, in the ragged end
TOKENS = [0, 1, 2, 7, 15, 16, 17, 30, 32, 37, 47, 48, 55, 63, 64, 90, 100, 112, 127, 128, 131, 140, 149, 144]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shared", [1, 2])
@pytest.mark.parametrize("g", [-5.0, -20.0, -60.0, -float("inf")])
def test_one_strong_decay_per_head(dtype, shared, g):
    """dg_t = <D, e^{g_t} S>, D the adjoint of the decayed state: off by at most what either is in its norm (6e-6 of both together in 32 bits, nine
    roundings to 16 bits), and by the decay's own rounding, 2^-23 |g|."""
    H = len(TOKENS)
    x = inputs(dtype, T=150, H=H, Hk=H // shared, dk=64, dv=64, seed=17)
    for h, t in enumerate(TOKENS):
        x["g"][0, t, h] = g
    got = host(run(x)["dg"])
    a = {k: host(v) for k, v in x.items()}
    for h, t in enumerate(TOKENS):
        if not np.isfinite(g):
            assert got[0, t, h] == 0.0, (h, t)
            continue
        y = {n: a[n][:, :, h // shared:h // shared + 1] for n in "qk"} | {n: a[n][:, :, h:h + 1] for n in ("v", "g", "beta")}
        states = gdr_oracle.forward(**y, S0=a["S0"][:, h:h + 1], scale=0.125, keep=True)["states"]
        decayed = np.exp(g) * states[t]
        tail = {n: v[:, t:].copy() for n, v in y.items()}
        tail["g"][:, 0] = 0.0
        D = gdr_oracle.backward(**tail, dO=a["dO"][:, t:, h:h + 1], S0=decayed, dS=a["dS"][:, h:h + 1], scale=0.125)["dS0"]
        want, scale = (D * decayed).sum(), np.linalg.norm(D) * np.linalg.norm(decayed)
        tol = (6e-6 if dtype == "f32" else 3 * 2.0 ** -8) + 2.0 ** -23 * abs(g)
        assert abs(got[0, t, h] - want) <= tol * scale, (h, t, got[0, t, h], want, scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [10.0, 1000.0])
def test_large_adjoints_of_the_final_states(dtype, size):
    """As exact relative to what they lead to as small ones."""
    from gdr_util import check, oracle
    x = inputs(dtype, B=2, T=200, H=4, Hk=2, dk=64, dv=128, seed=6)
    x["dS"] *= size
    check(run(x), oracle(x), dtype)
