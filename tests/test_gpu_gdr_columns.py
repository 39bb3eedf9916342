"""Gated delta rule where the scans take 32 columns a workgroup (more workgroups of 16 columns than CUs), over several chunks: a few of the
(sequence, head) pairs of a call against the fp64 oracle."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import check, inputs, oracle, run

pytestmark = pytest.mark.gpu


def part(x, seqs, key, cu=None):
    """The sequences `seqs` (packed: all) and the value heads of key head `key` of a call's tensors."""
    Hk = x["q"].shape[2] if "q" in x else x["dq"].shape[2]
    shared = (x["v"] if "v" in x else x["dv"]).shape[2] // Hk
    heads = slice(key * shared, (key + 1) * shared)
    rows = slice(None) if cu else seqs
    out = {}
    for n, t in x.items():
        if t is None:
            out[n] = None
        elif n in ("q", "k", "dq", "dk"):
            out[n] = t[rows, :, key:key + 1]
        elif n in ("S0", "dS", "S", "dS0"):
            out[n] = t[rows, heads]
        else:
            out[n] = t[rows, :, heads]
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("T", [200, 384])
def test_several_chunks(dtype, dk, dv, T):
    """72 or 40 pairs, 576 or 320 workgroups of 16 columns; with and without states, kept and formed again."""
    B = 9 if dv == 64 else 5
    x = inputs(dtype, B=B, T=T, H=8, Hk=4, dk=dk, dv=dv, seed=dk + T)
    for states in (False, True):
        want = {(b, key): oracle(part(x, slice(b, b + 1), key), states=states) for b, key in ((0, 0), (B // 2, 1), (B - 1, 3))}
        for keep in ((True, True), (False, False)):
            got = run(x, states=states, keep=keep)
            for (b, key), w in want.items():
                check(part(got, slice(b, b + 1), key), w, dtype, (states, keep, b, key))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 128)])
def test_packed(dtype, dk, dv):
    lens = [200, 64, 130, 1, 321]
    cu = np.cumsum([0] + lens).tolist()
    x = inputs(dtype, T=cu[-1], H=16, Hk=4, dk=dk, dv=dv, seqs=len(lens), seed=3)
    for states in (False, True):
        want = {key: oracle(part(x, None, key, cu), cu=cu, states=states) for key in (0, 3)}
        for keep in ((True, True), (False, False)):
            got = run(x, cu=cu, states=states, keep=keep)
            for key, w in want.items():
                check(part(got, None, key, cu), w, dtype, (states, keep, key))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 64)])
def test_one_long_sequence_among_short_ones(dtype, dk, dv):
    """More sequences than 16 columns are taken for where they are of equal lengths; by the longest one they are."""
    lens = [20] * 9 + [1500] + [1, 64, 70] * 4
    cu = np.cumsum([0] + lens).tolist()
    x = inputs(dtype, T=cu[-1], H=4, Hk=2, dk=dk, dv=dv, seqs=len(lens), seed=5)
    for states in (False, True):
        want = oracle(part(x, None, 1, cu), cu=cu, states=states)
        for keep in ((True, True), (False, False)):
            check(part(run(x, cu=cu, states=states, keep=keep), None, 1, cu), want, dtype, (states, keep))
