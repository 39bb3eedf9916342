"""The gated delta rule's backward split into segments of the sequence (two streams): bit for bit what one piece gives."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import check, inputs, oracle
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu
NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dS0")


@pytest.fixture
def segments():
    old = binding.set_segments(0)
    yield binding.set_segments
    binding.set_segments(old)


def forward(x, keep, states):
    return binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S0=x["S0"] if states else None, save_e=True, save_states=keep,
                                     save_operands=keep, output_final_state=False)


def backward(x, f, states, S0=None, **kw):
    return binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], x["dO"], S0=(x["S0"] if S0 is None else S0) if states else None,
                                     states=f["states"], operands=f["operands"], dS_final=x["dS"] if states else None, want_dS0=states, **kw)


def same(a, b):
    return all((a[n] is None and b[n] is None) or torch.equal(a[n], b[n]) for n in NAMES)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("states", [True, False])
def test_any_number_of_segments(segments, dtype, keep, states):
    x = inputs(dtype, B=2, T=1300, H=4, Hk=2, dk=64, dv=128, seed=3)
    f = forward(x, keep, states)
    segments(1)
    want = backward(x, f, states)
    check({n: want[n] for n in NAMES}, {n: w for n, w in oracle(x, states=states).items() if n in NAMES}, dtype)
    for k in (2, 3, 5, 16):
        segments(k)
        assert same(backward(x, f, states), want), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [255, 256, 512, 513])
def test_lengths_around_the_smallest_split(segments, dtype, T):
    x = inputs(dtype, T=T, H=3, Hk=1, dk=128, dv=64, seed=T)
    f = forward(x, False, True)
    segments(1)
    want = backward(x, f, True)
    segments(2)
    assert same(backward(x, f, True), want)


def test_packed_batches_are_not_split(segments):
    cu = [0, 300, 901, 1300]
    x = inputs("bf16", T=1300, H=4, Hk=4, dk=64, dv=64, seqs=3, seed=4)
    f = binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], cu_seqlens=cu, save_e=True, output_final_state=False)
    call = lambda: binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], x["dO"], cu_seqlens=cu)
    segments(1)
    want = call()
    segments(3)
    assert same(call(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_adjoints_written_over_the_states_that_are_read_beside(segments, dtype):
    """dS0 over S0, from which the second stream reconstructs the states meanwhile, and over dS_final."""
    x = inputs(dtype, T=1000, H=8, Hk=8, dk=128, dv=128, seed=6)
    f = forward(x, False, True)
    segments(1)
    want = backward(x, f, True)
    segments(3)
    S0 = x["S0"].clone()
    got = backward(x, f, True, S0=S0, out={"dS0": S0})
    assert torch.equal(S0, want["dS0"]) and same(got, want)
    x["dS"] = x["dS"].clone()
    assert same(backward(x, f, True, out={"dS0": x["dS"]}), want)


def test_captured_and_replayed(segments):
    segments(3)
    x = inputs("bf16", T=1000, H=4, Hk=2, dk=128, dv=128, seed=7)
    step = lambda y: backward(y, forward(y, False, True), True)
    step(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(x)
    for seed in (8, 9, 10):
        new = inputs("bf16", T=1000, H=4, Hk=2, dk=128, dv=128, seed=seed)
        for n in x:
            x[n].copy_(new[n])
        g.replay()
        torch.cuda.synchronize()
        want = step(new)
        torch.cuda.synchronize()
        assert same(got, want), seed


def test_two_streams_share_the_second_one(segments):
    segments(4)
    xs = [inputs("bf16", T=1500, H=4, Hk=4, dk=128, dv=128, seed=s) for s in (11, 12)]
    fs = [forward(x, False, True) for x in xs]
    want = [backward(x, f, True) for x, f in zip(xs, fs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(3):
        got = []
        for x, f, s in zip(xs, fs, streams):
            with torch.cuda.stream(s):
                got.append(backward(x, f, True))
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype,dk", [("f32", 64), ("bf16", 128)])
def test_the_librarys_own_choice(segments, dtype, dk):
    x = inputs(dtype, T=8192 if dtype == "bf16" else 4096, H=16, Hk=16, dk=dk, dv=dk, seed=13)
    f = forward(x, True, False)
    got = backward(x, f, False)
    segments(1)
    assert same(got, backward(x, f, False))
