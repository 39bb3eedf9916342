"""Inputs, oracle and tolerances of the gated delta rule's GPU tests."""
import math

import numpy as np
import torch

from gpu_util import host, rel_err, rms_rel_err
from oracle import gdr_oracle
from paper_2605_05838_amd import binding

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(dtype, B=1, T=64, H=2, Hk=2, dk=64, dv=64, seqs=None, seed=0, decay=0.1):
    """Tensors on the GPU: unit keys and queries, decays of exp(-decay softplus), states and adjoints of them per sequence."""
    r = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=r)
    unit = lambda *s: torch.nn.functional.normalize(n(*s), dim=-1)
    x = dict(q=unit(B, T, Hk, dk), k=unit(B, T, Hk, dk), v=n(B, T, H, dv), dO=n(B, T, H, dv))
    x = {k: v.to(DT[dtype]) for k, v in x.items()}
    seqs = seqs or B
    x.update(g=-decay * torch.nn.functional.softplus(n(B, T, H)), beta=torch.sigmoid(n(B, T, H)), S0=0.3 * n(seqs, H, dk, dv),
             dS=0.1 * n(seqs, H, dk, dv))
    return {k: v.cuda() for k, v in x.items()}


def oracle(x, cu=None, states=True, scale=None, backward=True):
    """The oracle's outputs for such inputs, packed sequences one by one."""
    a = {k: host(v) for k, v in x.items()}
    scale = a["q"].shape[-1] ** -0.5 if scale is None else scale
    T = a["q"].shape[1]
    parts = []
    for i, (t0, t1) in enumerate([(0, T)] if cu is None else zip(cu, cu[1:])):
        y = {k: a[k][:, t0:t1] for k in ("q", "k", "v", "g", "beta")}
        at = slice(None) if cu is None else slice(i, i + 1)
        S0, dS = (a["S0"][at], a["dS"][at]) if states else (None, None)
        p = gdr_oracle.forward(**y, S0=S0, scale=scale)
        if backward:
            p.update(gdr_oracle.backward(**y, dO=a["dO"][:, t0:t1], S0=S0, dS=dS, scale=scale))
        parts.append(p)
    return {k: np.concatenate([p[k] for p in parts], axis=0 if k in ("S", "dS0") else 1) for k in parts[0]}


# Roundings to 16 bits on the way to an output, each off by at most 2^-8, independent: they add in quadrature.
#   o: S, R, T (E), P, E, o;  dv: D, dE, T, dv and those of P^T's product;  e: S, R, T, e;  dq: S, W1, beta k, E, dV (in W), dq;
#   dk: S, dV, W1, W2, beta k, E, D, dk;  dg, dbeta: S, D, E, dV twice over, and the output
ROUNDINGS = {"o": 6, "e": 4, "dv": 5, "dq": 6, "dk": 8, "dg": 9, "dbeta": 9}


def tolerance(name, dtype):
    """Bound of the rms-relative error."""
    if dtype == "f32":
        # ten products of up to 128 terms follow one another, every term and every sum off by 2^-24 at random: sqrt(2 * 10 * 128) 2^-24 = 3e-6,
        # and twice that for sums whose terms cancel
        return 6e-6
    if name in ("S", "dS0"):
        # value + remainder: 2^-16 at most each, of S, T, R, E (D, P, T, dE, dV, dO)
        return math.sqrt(6) * 2.0 ** -16
    return math.sqrt(ROUNDINGS[name]) * 2.0 ** -8


def check(got, want, dtype, what=""):
    errs = {}
    for name, w in want.items():
        if got.get(name) is None:
            continue
        g = host(got[name])
        assert g.shape == w.shape, (name, g.shape, w.shape)
        assert np.isfinite(g).all(), (what, name)
        scale = np.sqrt(np.mean(np.square(w)))
        if scale == 0:
            assert not g.any(), (what, name)
            continue
        errs[name] = (rms_rel_err(g, w), tolerance(name, dtype), rel_err(g, w))
    print(what, {k: "%.1e/%.1e max %.1e" % v for k, v in errs.items()}, flush=True)
    bad = {k: v for k, v in errs.items() if not (v[0] <= v[1] and v[2] <= 8 * v[1])} # (an element: 8 times the rms)
    assert not bad, (what, bad)


def run(x, cu=None, states=True, keep=(True, True), backward=True, scale=None):
    S0, dS = (x["S0"], x["dS"]) if states else (None, None)
    f = binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S0=S0, scale=scale, cu_seqlens=cu, save_e=True,
                                  save_states=keep[0], save_operands=keep[1], output_final_state=states)
    out = {k: f[k] for k in ("o", "S", "e")}
    if backward:
        b = binding.mdn_gdr_chunk_bwd(x["q"], x["k"], x["g"], x["beta"], f["e"], x["dO"], S0=S0, states=f["states"], operands=f["operands"],
                                      dS_final=dS, scale=scale, cu_seqlens=cu, want_dS0=states)
        out.update((k, b[k]) for k in ("dq", "dk", "dv", "dg", "dbeta", "dS0"))
    return out
