"""The gated delta rule and the 8-bit checkpoints as a layer uses them, in one run: forward with checkpoints, backward from them."""
import numpy as np
import pytest
import torch

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import DT, check as check_rule, inputs, oracle
from gpu_util import host, rel_err
from oracle import kept_oracle
from oracle import layer_ops_oracle as lo
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu


def layer_inputs(dtype, B, T, H, d, seed=0):
    r = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=r)
    x = {k: n(B, T, H, d).to(DT[dtype]).cuda() for k in ("x_q", "x_k", "x_v", "gate", "dy")}
    x.update(g=(-0.1 * torch.nn.functional.softplus(n(B, T, H))).cuda(), beta=torch.sigmoid(n(B, T, H)).cuda(),
             d=(0.3 * torch.rand(H, generator=r)).cuda(), w=(torch.rand(d, generator=r) + 0.5).cuda())
    return x


def step(x, cu=None):
    """What a training step of the layer keeps between the two halves: the checkpoints, e and the states."""
    f = binding.mdn_frontend_fwd_keep(x["x_q"], x["x_k"], x["x_v"], x["d"])
    c = binding.mdn_gdr_chunk_fwd(f["q"], f["k"], f["v"], x["g"], x["beta"], cu_seqlens=cu, save_e=True, save_states=True, output_final_state=False)
    y = binding.mdn_epilogue_fwd_keep(c["o"], x["gate"], x["w"])
    be = binding.mdn_epilogue_bwd_kept(y["kept_o"], y["kept_g"], x["w"], x["dy"])
    kept = [f["kept_" + n] for n in "qkv"]
    again = binding.mdn_frontend_fwd_kept(*kept, x["d"], x["dy"].dtype)
    b = binding.mdn_gdr_chunk_bwd(again["q"], again["k"], x["g"], x["beta"], c["e"], be["do"], states=c["states"], cu_seqlens=cu)
    bf = binding.mdn_frontend_bwd_kept(*kept, x["d"], b["dq"], b["dk"], b["dv"])
    return f, c, y, be, again, b, bf


def flat(parts):
    return [t for p in parts for k, v in p.items() if v is not None and k != "workspace" for t in (v if isinstance(v, tuple) else (v,))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cu", [None, [0, 1, 70, 150]])
def test_every_stage_of_a_step(dtype, cu):
    """Each stage against its oracle at the values that the stage before handed to it."""
    x = layer_inputs(dtype, 1, 150, 4, 64)
    f, c, y, be, again, b, bf = step(x, cu)
    tol = 1e-5 if dtype == "f32" else 2.0 ** -8
    a = {k: host(v) for k, v in x.items()}
    vals = {n: kept_oracle.values(a["x_" + n]) for n in "qkv"}
    want = lo.frontend_forward(a["x_q"], a["x_k"], a["x_v"], a["d"])
    want_again = lo.frontend_forward(vals["q"], vals["k"], vals["v"], a["d"])
    for n in "qkv":
        assert rel_err(host(f[n]), want[n]) <= tol and rel_err(host(again[n]), want_again[n]) <= tol
    z = torch.zeros(3 if cu else 1, 4, 64, 64, device="cuda")
    rule = dict(q=f["q"], k=f["k"], v=f["v"], g=x["g"], beta=x["beta"], dO=be["do"], S0=z, dS=z)
    check_rule({"o": c["o"], "e": c["e"]}, {k: v for k, v in oracle(rule, cu=cu).items() if k in ("o", "e")}, dtype, "forward")
    vo, vg = kept_oracle.values(host(c["o"])), kept_oracle.values(a["gate"])
    assert rel_err(host(y["y"]), lo.epilogue_forward(host(c["o"]), a["gate"], a["w"])) <= tol
    w = lo.epilogue_backward(vo, vg, a["w"], a["dy"])
    assert rel_err(host(be["do"]), w["do"]) <= tol and rel_err(host(be["dg"]), w["dg"]) <= tol and rel_err(host(be["dw"]), w["dw"]) <= 1e-5
    w = lo.frontend_backward(vals["q"], vals["k"], vals["v"], a["d"], host(b["dq"]), host(b["dk"]), host(b["dv"]))
    for n in ("dx_q", "dx_k", "dx_v"):
        assert rel_err(host(bf[n]), w[n]) <= tol


def test_the_gradients_are_near_those_without_checkpoints():
    """A kept value is off by at most 2^-7 of its block's largest one, 2.2 standard deviations: 2^-7 * 2.2 / sqrt(3) = 1 % of a typical one at
    random; a gradient depends on three such tensors and the two of the back end, each entering more than once: 5 * 1 % * 2."""
    x = layer_inputs("f32", 2, 200, 4, 64, seed=4)
    _, _, _, be, _, b, bf = step(x)
    p = binding.mdn_frontend_fwd(x["x_q"], x["x_k"], x["x_v"], x["d"])
    c = binding.mdn_gdr_chunk_fwd(p["q"], p["k"], p["v"], x["g"], x["beta"], save_e=True)
    e = binding.mdn_epilogue_bwd(c["o"], x["gate"], x["w"], x["dy"])
    r = binding.mdn_gdr_chunk_bwd(p["q"], p["k"], x["g"], x["beta"], c["e"], e["do"])
    rf = binding.mdn_frontend_bwd(x["x_q"], x["x_k"], x["x_v"], x["d"], r["dq"], r["dk"], r["dv"])
    for got, want in [(be["do"], e["do"]), (be["dg"], e["dg"]), (be["dw"], e["dw"])] + [(b[n], r[n]) for n in ("dv", "dg", "dbeta")] + \
            [(bf[n], rf[n]) for n in ("dx_q", "dx_k", "dx_v", "dd")]:
        err = float((got - want).norm() / want.norm())
        assert 0 < err < 0.1, err


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cu", [None, [0, 3, 131, 200]])
def test_a_captured_step_replays(dtype, cu):
    """Captured once, replayed with other inputs and other work between the replays: every replay is the eager result bit for bit."""
    x = layer_inputs(dtype, 1, 200, 4, 128, seed=1)
    step(x, cu)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = flat(step(x, cu))
    for seed in (2, 3, 4):
        new = layer_inputs(dtype, 1, 200, 4, 128, seed=seed)
        for k in x:
            x[k].copy_(new[k])
        g.replay()
        torch.cuda.synchronize()
        want = flat(step(new, cu))
        torch.cuda.synchronize()
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_two_streams_at_once():
    """Calls on two streams of their own, none ordered with the other, each with its own workspace: bit for bit what they give alone."""
    xs = [layer_inputs("bf16", 2, 500, 8, 128, seed=s) for s in (5, 6)]
    want = [flat(step(x)) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(3):
        got = []
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append(flat(step(x)))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_states_in_place_and_buffers_reused(dtype):
    """S_final over S0, dS0 over S0 or dS_final; the tensors of an earlier call, filled with NaN, as outputs and workspace."""
    x = inputs(dtype, B=2, T=100, H=4, Hk=2, dk=64, dv=128, seed=8)
    fwd = lambda S0, **kw: binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S0=S0, save_e=True, **kw)
    bwd = lambda S0, dS, **kw: binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], x["dO"], S0=S0, dS_final=dS, want_dS0=True, **kw)
    f = fwd(x["S0"])
    S = x["S0"].clone()
    o = fwd(S, out={"S": S})
    assert o["S"] is S or o["S"].data_ptr() == S.data_ptr()
    assert torch.equal(S, f["S"]) and torch.equal(o["o"], f["o"])
    b = bwd(x["S0"], x["dS"])
    for over in ("S0", "dS"):
        y = {k: x[k].clone() for k in ("S0", "dS")}
        c = bwd(y["S0"], y["dS"], out={"dS0": y[over]})
        assert torch.equal(y[over], b["dS0"]) and all(torch.equal(c[k], b[k]) for k in ("dq", "dk", "dv", "dg", "dbeta"))
    for t in b.values():
        t.fill_(float("nan")) if t.is_floating_point() else t.fill_(255)
    again = bwd(x["S0"], x["dS"], workspace=b["workspace"], out=b)
    want = bwd(x["S0"], x["dS"])
    assert all(again[k].data_ptr() == b[k].data_ptr() and torch.equal(again[k], want[k]) for k in ("dq", "dk", "dv", "dg", "dbeta", "dS0"))
