"""Gated delta rule on the GPU against its fp64 oracle."""
import numpy as np
import pytest
import torch

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import DT, check, inputs, oracle, run
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_one_chunk(dtype, dk, dv):
    x = inputs(dtype, T=64, dk=dk, dv=dv, seed=dk + dv)
    check(run(x, states=False), oracle(x, states=False), dtype, "no states")
    check(run(x), oracle(x), dtype, "states")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 15, 63, 65, 128, 130, 250])
def test_lengths(dtype, T):
    x = inputs(dtype, B=2, T=T, H=3, Hk=3, dk=128, dv=64, seed=T)
    check(run(x, states=False), oracle(x, states=False), dtype, "no states")
    check(run(x), oracle(x), dtype, "states")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keep", [(False, False), (True, False), (False, True)])
def test_what_the_forward_did_not_keep_is_formed_again(dtype, keep):
    """Operands bit for bit (a call with dS0 forms them in any case); states from e as it was kept, rounded to the storage type, where the
    forward went on from 32 bits: the same to the tolerance, and bit for bit without 16-bit storage."""
    x = inputs(dtype, B=1, T=300, H=4, Hk=2, dk=64, dv=128, seed=5)
    for states in (False, True):
        a, b = run(x, states=states), run(x, states=states, keep=keep)
        check(b, oracle(x, states=states), dtype)
        for name in a if dtype == "f32" or keep[0] else ("o", "S", "e", "dv", "dS0"):
            assert (a[name] is None and b[name] is None) or torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk", [(4, 1), (6, 2), (16, 16)])
def test_shared_key_heads(dtype, H, Hk):
    x = inputs(dtype, B=2, T=140, H=H, Hk=Hk, dk=128, dv=128, seed=H)
    check(run(x), oracle(x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[1], [5, 64, 1, 130, 65], [1] * 40, [200, 3, 3, 90]])
def test_packed(dtype, lens):
    cu = np.cumsum([0] + lens).tolist()
    x = inputs(dtype, T=cu[-1], H=4, Hk=2, dk=64, dv=64, seqs=len(lens), seed=len(lens))
    check(run(x, cu=cu, states=False), oracle(x, cu=cu, states=False), dtype, "no states")
    check(run(x, cu=cu), oracle(x, cu=cu), dtype, "states")
    check(run(x, cu=cu, keep=(False, False)), oracle(x, cu=cu), dtype, "nothing kept")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_sequences_than_a_table_launch_holds(dtype):
    lens = [1 + i % 3 for i in range(300)]
    cu = np.cumsum([0] + lens).tolist()
    x = inputs(dtype, T=cu[-1], H=2, Hk=1, dk=64, dv=64, seqs=len(lens), seed=9)
    check(run(x, cu=cu), oracle(x, cu=cu), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_at_their_limits(dtype):
    """Decays of 0 (log -inf), of next to nothing, of exactly 1; step sizes of 0 and 1."""
    x = inputs(dtype, B=1, T=200, H=4, Hk=4, dk=64, dv=64, seed=11)
    x["g"][:, 20, 0] = -float("inf")
    x["g"][:, 70:90, 1] = -40.0
    x["g"][:, 100, 1] = -1e30
    x["g"][:, :, 2] = 0.0
    x["beta"][:, 30:60, 3] = 0.0
    x["beta"][:, 60:90, 3] = 1.0
    check(run(x), oracle(x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_strong_decay_leaves_the_tokens_behind_it_exact(dtype):
    """The sums of the log decays run to thousands; what counts between two later tokens is their difference."""
    x = inputs(dtype, B=1, T=64, H=2, Hk=2, dk=64, dv=64, seed=12, decay=0.01)
    x["g"][:, 5:30] = -90.0
    check(run(x), oracle(x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,Hk,dk,dv", [(1, 1, 2, 2, 64, 64), (3, 1, 6, 2, 128, 64), (2, 7, 4, 4, 64, 128), (300, 1, 4, 1, 128, 128),
                                            (2, 66, 2, 1, 128, 128)])
def test_step(dtype, B, T, H, Hk, dk, dv):
    x = inputs(dtype, B=B, T=T, H=H, Hk=Hk, dk=dk, dv=dv, seed=B + T)
    want = oracle(x, backward=False)
    S = x["S0"].clone()
    o = binding.mdn_gdr_recurrent_step(x["q"], x["k"], x["v"], x["g"], x["beta"], S)
    err = lambda a, b: np.linalg.norm(a.double().cpu().numpy() - b) / np.linalg.norm(b)
    # fp32 throughout: sums of 128 terms, T of them one after the other; o is rounded once more
    assert err(S, want["S"]) < 2e-6 and err(o, want["o"]) < (3e-6 if dtype == "f32" else 2.0 ** -8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefill_goes_over_into_steps(dtype):
    x = inputs(dtype, B=2, T=150, H=4, Hk=2, dk=128, dv=128, seed=21)
    whole = oracle(x, backward=False)
    head = {k: (v[:, :137].contiguous() if v.dim() > 2 and k not in ("S0", "dS") else v) for k, v in x.items()}
    f = binding.mdn_gdr_chunk_fwd(head["q"], head["k"], head["v"], head["g"], head["beta"], S0=x["S0"])
    tail = {k: x[k][:, 137:].contiguous() for k in ("q", "k", "v", "g", "beta")}
    o = binding.mdn_gdr_recurrent_step(*tail.values(), f["S"])
    check({"o": torch.cat((f["o"], o), 1), "S": f["S"]}, {k: whole[k] for k in ("o", "S")}, dtype)
