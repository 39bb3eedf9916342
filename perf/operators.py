"""The gated delta rule (chunked with its gradients, and token by token) and the 8-bit checkpoints of the layer's inputs, as cases that
can be timed and compared: in their plain form on torch tensors, and through the functions of `paper_2605_05838_amd.binding`.

    S_t = e^{g_t} S_{t-1} + beta_t k_t e_t^T,    e_t = v_t - e^{g_t} S_{t-1}^T k_t,    o_t = scale S_t^T q_t

Value head h reads key head h // (H / Hk).  Shapes: the layer shapes of `synth.CONFIGS` and of the workloads of `bench.py` (2 to 16 heads of
64 or 128, up to 32 768 tokens), and odd lengths.
"""
import math
import random

import torch

own = False

CHUNK = 64
EPS = 1e-6


def listed():
    return [
        # one sequence being generated, one token per call: the smallest call there is, all latency
        dict(name="step_one", kind="step", B=1, T=1, H=16, Hk=16, dk=128, dv=128, dtype="bf16"),
        # a full serving batch, one token per sequence and call: 256 MB of states in and out
        dict(name="step_batch", kind="step", B=256, T=1, H=16, Hk=8, dk=128, dv=128, dtype="bf16"),
        # a few drafted tokens of each sequence taken at once, 32-bit storage
        dict(name="step_draft", kind="step", B=12, T=5, H=8, Hk=4, dk=64, dv=128, dtype="f32"),
        # one prompt of ordinary, odd length before its decoding starts (time to first token)
        dict(name="prefill_prompt", kind="prefill", B=1, T=777, H=16, Hk=16, dk=128, dv=128, n=0, carry=False, lens=0, dtype="bf16"),
        # a batch of equal prompts / an evaluation forward at the 400M layer shape
        dict(name="prefill_batch", kind="prefill", B=8, T=2048, H=8, Hk=8, dk=128, dv=128, n=0, carry=False, lens=0, dtype="bf16"),
        # prompts of mixed lengths packed into one call, going on from states they already have, four value heads to a key head
        dict(name="prefill_packed", kind="prefill", B=1, T=16384, H=16, Hk=4, dk=128, dv=128, n=24, carry=True, lens=1, dtype="bf16"),
        # the training step of the 1.3B layer shape, forward keeping what the backward can use
        dict(name="train_layer_shape", kind="train", B=4, T=4096, H=16, Hk=16, dk=128, dv=128, n=0, lens=0, keep=True, segment=False,
             dtype="bf16"),
        # training on one long document
        dict(name="train_long", kind="train", B=1, T=32768, H=16, Hk=16, dk=128, dv=128, n=0, lens=0, keep=True, segment=False,
             dtype="bf16"),
        # one segment of a longer sequence of odd length, shared key heads: states in, adjoints of the final states in, only e kept
        dict(name="train_segment", kind="train", B=3, T=1500, H=8, Hk=2, dk=64, dv=128, n=0, lens=0, keep=False, segment=True,
             dtype="bf16"),
        # 32-bit storage, small: how a model is checked against a reference before it is trained
        dict(name="train_f32", kind="train", B=2, T=1024, H=4, Hk=4, dk=64, dv=64, n=0, lens=0, keep=True, segment=False, dtype="f32"),
        # the elementwise operations around the rule with 8-bit checkpoints, forward and backward: one sequence of odd length
        dict(name="kept_sequence", kind="kept", B=1, T=777, H=16, d=128, dtype="bf16"),
        # the same at the 1.3B layer shape
        dict(name="kept_layer_shape", kind="kept", B=4, T=4096, H=16, d=128, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("step", "prefill", "prefill", "train", "train", "kept"))
    H = rng.choice((2, 4, 8, 16))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    # (token, head) pairs of a case: the fp32 matrix rate is a sixteenth of the bf16 one
    most = 16384 if dtype == "f32" else 262144
    if kind == "kept":
        B = rng.randint(1, 4)
        return dict(kind=kind, B=B, T=_log(rng, 1, 262144 // (2 if dtype == "f32" else 1) // (B * H)), H=H, d=rng.choice((64, 128)), dtype=dtype)
    Hk, dk, dv = H // rng.choice((1, 1, 2)), rng.choice((64, 128, 128)), rng.choice((64, 128, 128))
    if kind == "step":
        return dict(kind=kind, B=_log(rng, 1, 256), T=rng.choice((1, 1, 1, 2, 4, 7)), H=H, Hk=Hk, dk=dk, dv=dv, dtype=dtype)
    packed = rng.random() < 0.35
    B = 1 if packed else rng.randint(1, 8)
    T = _log(rng, 256 if packed else 1, min(32768, most // (B * H)))
    n = _log(rng, 2, max(3, min(48, T // 24))) if packed else 0
    lens = rng.randint(1, 10 ** 6) if packed else 0
    if kind == "prefill":
        return dict(kind=kind, B=B, T=T, H=H, Hk=Hk, dk=dk, dv=dv, n=n, carry=rng.random() < 0.5, lens=lens, dtype=dtype)
    return dict(kind=kind, B=B, T=T, H=H, Hk=Hk, dk=dk, dv=dv, n=n, lens=lens, keep=rng.random() < 0.6, segment=rng.random() < 0.4, dtype=dtype)


def _offsets(case):
    """Cumulative offsets of n sequences of log-normal lengths, at least one token each, T tokens together."""
    T, n = case["T"], case["n"]
    rnd = random.Random(case["lens"])
    w = [rnd.lognormvariate(0.0, 0.8) for _ in range(n)]
    total, acc, cu = sum(w), 0.0, [0]
    for i in range(n):
        acc += w[i]
        cu.append(min(max(cu[-1] + 1, int(round(acc / total * T))), T - (n - 1 - i)))
    cu[-1] = T
    return cu


class _Inputs:
    """Random tensors on the GPU from one seed, with the distributions of the path."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(self, *shape):
        return torch.randn(shape, device="cuda", generator=self.g)

    def values(self, *shape):
        return self.normal(*shape).to(self.dt)

    def unit(self, *shape):
        x = self.normal(*shape)
        return (x / x.norm(dim=-1, keepdim=True)).to(self.dt)


def prepare(case, seed):
    kind, B, T, H = case["kind"], case["B"], case["T"], case["H"]
    r = _Inputs(seed, case["dtype"])
    s = {"kind": kind}
    if kind == "kept":
        d = case["d"]
        # the short convolutions' outputs, the rule's output, the gate projection, and the adjoints that come back
        for name in ("x_q", "x_k", "x_v", "o", "g", "dy", "dq", "dk", "dv"):
            s[name] = r.values(B, T, H, d)
        s["d"] = 0.3 * torch.sigmoid(r.normal(H))
        s["w"] = 1.0 + 0.1 * r.normal(d)
        return s
    Hk, dk, dv = case["Hk"], case["dk"], case["dv"]
    s["scale"] = dk ** -0.5
    s["q"], s["k"], s["v"] = r.unit(B, T, Hk, dk), r.unit(B, T, Hk, dk), r.values(B, T, H, dv)
    s["g"] = -0.1 * torch.nn.functional.softplus(r.normal(B, T, H))   # decays around 0.93 a token
    s["beta"] = torch.sigmoid(r.normal(B, T, H))
    if kind == "step":
        s["S"], s["o"] = 0.3 * r.normal(B, H, dk, dv), None
        return s
    s["cu"] = _offsets(case) if case["n"] else None
    seqs = case["n"] or B
    if kind == "prefill":
        s["S0"] = 0.3 * r.normal(seqs, H, dk, dv) if case["carry"] else None
        s["f"] = {}
        return s
    s["dO"], s["keep"], s["segment"] = r.values(B, T, H, dv), case["keep"], case["segment"]
    s["S0"], s["dS"] = (0.3 * r.normal(seqs, H, dk, dv), 0.1 * r.normal(seqs, H, dk, dv)) if case["segment"] else (None, None)
    s["f"], s["b"] = {}, {}
    return s


# ---- the plain forms

def _rows(x, cu):
    """[1, T, ...] of packed sequences -> [n, longest, ...], zeros behind each; [B, T, ...] as it is."""
    if cu is None:
        return x
    longest = max(b - a for a, b in zip(cu, cu[1:]))
    at = torch.arange(longest, device=x.device)[None] + torch.tensor(cu[:-1], device=x.device)[:, None]
    real = at < torch.tensor(cu[1:], device=x.device)[:, None]
    y = x[0][at.clamp(max=x.shape[1] - 1)]
    return torch.where(real.reshape(real.shape + (1,) * (y.dim() - 2)), y, torch.zeros((), dtype=y.dtype, device=y.device))


def _packed(y, cu):
    """The reverse of _rows."""
    if cu is None:
        return y
    lens = torch.tensor([b - a for a, b in zip(cu, cu[1:])], device=y.device)
    real = torch.arange(y.shape[1], device=y.device)[None] < lens[:, None]
    return y[real][None]


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular A, from inverses of the diagonal blocks of half the size."""
    n = A.shape[-1]
    if n == 1:
        return torch.ones_like(A)
    h = n // 2
    blocks = _inverse(torch.stack((A[..., :h, :h], A[..., h:, h:])))
    low = -blocks[1] @ (A[..., h:, :h] @ blocks[0])
    top = torch.cat((blocks[0], torch.zeros_like(low).transpose(-1, -2)), -1)
    return torch.cat((top, torch.cat((low, blocks[1]), -1)), -2)


def _rule(q, k, v, g, beta, S, scale):
    """Chunks of 64 tokens, [B, T, H, d] and states [B, H, dk, dv] in 32 bits -> o and the final states."""
    B, T, H, _ = v.shape
    N = -(-T // CHUNK)

    def split(x):   # [B, T, H, ...] -> [B, H, N, 64, ...]
        x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, N * CHUNK - T))
        return x.reshape(B, N, CHUNK, *x.shape[2:]).permute(0, 3, 1, 2, *range(4, x.dim() + 1))

    shared = H // q.shape[2]
    q, k, v = (split(x) for x in (q.repeat_interleave(shared, 2), k.repeat_interleave(shared, 2), v))
    g, beta = split(g[..., None])[..., 0], split(beta[..., None])[..., 0]
    G = g.double().cumsum(-1)
    low = torch.ones(CHUNK, CHUNK, device=q.device).tril().bool()
    c = torch.where(low, G[..., :, None] - G[..., None, :], torch.zeros((), device=q.device, dtype=G.dtype)).exp().float()
    c = torch.where(low, c * beta[..., None, :], torch.zeros((), device=q.device))
    Tm = _inverse((c * (k @ k.transpose(-1, -2))).tril(-1))
    P = c * (q @ k.transpose(-1, -2))
    from_start, to_end, whole = G.exp().float()[..., None], (G[..., -1:] - G).exp().float(), G[..., -1].exp().float()
    kS, qS, kE = k * from_start, q * from_start, k * (to_end * beta)[..., None]
    o = []
    for n in range(N):
        E = Tm[:, :, n] @ (v[:, :, n] - kS[:, :, n] @ S)
        o.append(qS[:, :, n] @ S + P[:, :, n] @ E)
        S = whole[:, :, n, None, None] * S + kE[:, :, n].transpose(-1, -2) @ E
    return scale * torch.stack(o, 2).permute(0, 2, 3, 1, 4).reshape(B, N * CHUNK, H, -1)[:, :T], S


def _plain_chunked(s):
    train, cu, dt = s["kind"] == "train", s["cu"], s["q"].dtype
    leaves = {k: s[k].detach().float().requires_grad_(train) for k in ("q", "k", "v", "g", "beta")}
    seqs = len(cu) - 1 if cu else s["v"].shape[0]
    if s["S0"] is None:
        S0 = torch.zeros(seqs, s["v"].shape[2], s["q"].shape[-1], s["v"].shape[-1], device=s["q"].device)
    else:
        S0 = s["S0"].detach().requires_grad_(train)
    with torch.set_grad_enabled(train):
        o, S = _rule(*(_rows(leaves[k], cu) for k in ("q", "k", "v", "g", "beta")), S0, s["scale"])
        o = _packed(o, cu)
    if not train:
        return {"o": o.to(dt), "S": S}
    out = {"o": o.detach().to(dt)}
    wrt = list(leaves.values()) + ([S0] if s["segment"] else [])
    grads = torch.autograd.grad((o, S) if s["segment"] else (o,), wrt, (s["dO"].float(), s["dS"]) if s["segment"] else (s["dO"].float(),))
    out.update(("d" + k, x.to(dt)) for k, x in zip(leaves, grads))
    if s["segment"]:
        out["S"], out["dS0"] = S.detach(), grads[-1]
    return out


def _plain_step(s):
    S, dt = s["S"], s["q"].dtype
    q, k, v = (s[x].float() for x in ("q", "k", "v"))
    shared = v.shape[2] // q.shape[2]
    q, k, a = q.repeat_interleave(shared, 2), k.repeat_interleave(shared, 2), s["g"].exp()
    o = []
    for t in range(v.shape[1]):
        S = a[:, t, :, None, None] * S
        e = v[:, t] - (S * k[:, t, :, :, None]).sum(-2)
        S = S + (s["beta"][:, t, :, None] * k[:, t])[..., None] * e[..., None, :]
        o.append(s["scale"] * (S * q[:, t, :, :, None]).sum(-2))
    s["S"].copy_(S)
    return {"o": torch.stack(o, 1).to(dt), "S": s["S"]}


def _kept(x):
    """What an 8-bit checkpoint of x stands for: blocks of 32 with a power-of-two step of 2^-6 of the largest value's power of two."""
    b = x.float().reshape(*x.shape[:-1], -1, 32)
    e = torch.frexp(b.abs().amax(-1, keepdim=True))[1] - 7
    step = ((e.clamp(min=-126).int() + 127) << 23).view(torch.float32)   # 2^e, by its bits: exactly
    return ((b / step).round().clamp(-127, 127) * step).reshape(x.shape)


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _front(x_q, x_k, x_v, d):
    q, k, v = (x * _sigmoid(x) for x in (x_q, x_k, x_v))
    q = q - d[:, None] * k
    return tuple(x * torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS) for x in (q, k)) + (v,)


def _plain_kept(s):
    dt, d, w = s["o"].dtype, s["d"], s["w"]
    x = tuple(s[n].float() for n in ("x_q", "x_k", "x_v"))
    out = dict(zip(("q", "k", "v"), _front(*x, d)))
    o, g = s["o"].float(), s["g"].float()
    out["y"] = _sigmoid(g) * w * o * torch.rsqrt((o * o).mean(-1, keepdim=True) + EPS)
    # backward, from the checkpoints: the back end
    o, g, dy = _kept(s["o"]), _kept(s["g"]), s["dy"].float()
    ir, sg = torch.rsqrt((o * o).mean(-1, keepdim=True) + EPS), _sigmoid(g)
    n = o * ir
    dn = dy * sg * w
    out["do"] = (dn - n * (n * dn).mean(-1, keepdim=True)) * ir
    out["dg"] = dn * n * (1.0 - sg)
    dw = (dy * sg * n).double().sum((0, 1, 2)).float()
    # the front end: its outputs again, and its adjoint
    x = tuple(_kept(s[n]) for n in ("x_q", "x_k", "x_v"))
    again = _front(*x, d)
    out.update(zip(("q_again", "k_again", "v_again"), again))
    sig = [_sigmoid(t) for t in x]
    slope = [a * (1.0 + t * (1.0 - a)) for t, a in zip(x, sig)]
    ks = x[1] * sig[1]
    qc = x[0] * sig[0] - d[:, None] * ks
    iq, ik = (torch.rsqrt((t * t).sum(-1, keepdim=True) + EPS) for t in (qc, ks))
    dq, dk, dv = (s[n].float() for n in ("dq", "dk", "dv"))
    dqc = (dq - again[0] * (again[0] * dq).sum(-1, keepdim=True)) * iq
    dks = (dk - again[1] * (again[1] * dk).sum(-1, keepdim=True)) * ik - d[:, None] * dqc
    out["dx_q"], out["dx_k"], out["dx_v"] = dqc * slope[0], dks * slope[1], dv * slope[2]
    dd = -(dqc * ks).double().sum((0, 1, 3)).float()
    return {**{k: v.to(dt) for k, v in out.items()}, "dw": dw, "dd": dd}


# ---- the framework's calls

def _own_step(s):
    from paper_2605_05838_amd import binding
    s["o"] = binding.mdn_gdr_recurrent_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["S"], scale=s["scale"], out=s["o"])
    return {"o": s["o"], "S": s["S"]}


def _own_prefill(s):
    from paper_2605_05838_amd import binding
    f = s["f"] = binding.mdn_gdr_chunk_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], S0=s["S0"], scale=s["scale"], cu_seqlens=s["cu"],
                                           workspace=s["f"].get("workspace"), out=s["f"])
    return {"o": f["o"], "S": f["S"]}


def _own_train(s):
    from paper_2605_05838_amd import binding
    keep, seg = s["keep"], s["segment"]
    f = s["f"] = binding.mdn_gdr_chunk_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], S0=s["S0"], scale=s["scale"], cu_seqlens=s["cu"],
                                           save_e=True, save_states=keep, save_operands=keep, output_final_state=seg,
                                           workspace=s["f"].get("workspace"), out=s["f"])
    b = s["b"] = binding.mdn_gdr_chunk_bwd(s["q"], s["k"], s["g"], s["beta"], f["e"], s["dO"], S0=s["S0"], states=f["states"],
                                           operands=f["operands"], dS_final=s["dS"], scale=s["scale"], cu_seqlens=s["cu"], want_dS0=seg,
                                           workspace=s["b"].get("workspace"), out=s["b"])
    out = {"o": f["o"], **{k: b[k] for k in ("dq", "dk", "dv", "dg", "dbeta")}}
    if seg:
        out["S"], out["dS0"] = f["S"], b["dS0"]
    return out


def _own_kept(s):
    from paper_2605_05838_amd import binding
    f = binding.mdn_frontend_fwd_keep(s["x_q"], s["x_k"], s["x_v"], s["d"], eps=EPS)
    e = binding.mdn_epilogue_fwd_keep(s["o"], s["g"], s["w"], eps=EPS)
    be = binding.mdn_epilogue_bwd_kept(e["kept_o"], e["kept_g"], s["w"], s["dy"], eps=EPS)
    kept = (f["kept_q"], f["kept_k"], f["kept_v"])
    again = binding.mdn_frontend_fwd_kept(*kept, s["d"], dtype=s["o"].dtype, eps=EPS)
    bf = binding.mdn_frontend_bwd_kept(*kept, s["d"], s["dq"], s["dk"], s["dv"], eps=EPS)
    out = {"q": f["q"], "k": f["k"], "v": f["v"], "y": e["y"], "do": be["do"], "dg": be["dg"]}
    out.update((x + "_again", again[x]) for x in ("q", "k", "v"))
    out.update((x, bf[x]) for x in ("dx_q", "dx_k", "dx_v"))
    return {**out, "dw": be["dw"], "dd": bf["dd"]}


def run(state):
    kind = state["kind"]
    if own:
        return {"step": _own_step, "prefill": _own_prefill, "train": _own_train, "kept": _own_kept}[kind](state)
    return {"step": _plain_step, "prefill": _plain_chunked, "train": _plain_chunked, "kept": _plain_kept}[kind](state)


def work(case):
    """Bytes: every tensor of the call once (what passes between forward and backward is not counted, except the 8-bit checkpoints).
    Operations: per token and value head, the chunkwise algorithm at 64 tokens a chunk (forward 6 dk dv + 2 C dk + C dv, backward 12 dk dv +
    6 C dk + 3 C dv: triangles by halves), for the step the recurrence itself (7 dk dv)."""
    kind, B, T, H = case["kind"], case["B"], case["T"], case["H"]
    es, C, n = (2 if case["dtype"] == "bf16" else 4), CHUNK, B * T * H
    if kind == "kept":
        d = case["d"]
        kept = d + d // 32
        # x_q, x_k, x_v, o, g, dy, dq, dk, dv in; q, k, v, y, do, dg, the three again, dx_q, dx_k, dx_v out; five checkpoints out and in
        return {"bytes": n * (21 * d * es + 10 * kept), "flops": 250 * n * d}
    Hk, dk, dv = case["Hk"], case["dk"], case["dv"]
    keys, vals, gates = B * T * Hk * dk * es, n * dv * es, 8 * n
    state = 4 * H * dk * dv
    if kind == "step":
        return {"bytes": 2 * keys + 2 * vals + gates + 2 * B * state, "flops": 7 * dk * dv * n}
    seqs = case["n"] or B
    fwd, bwd = n * (6 * dk * dv + 2 * C * dk + C * dv), n * (12 * dk * dv + 6 * C * dk + 3 * C * dv)
    if kind == "prefill":
        return {"bytes": 2 * keys + 2 * vals + gates + seqs * state * (2 if case["carry"] else 1), "flops": fwd}
    return {"bytes": 4 * keys + 4 * vals + gates + 2 * es * n + (4 * seqs * state if case["segment"] else 0), "flops": fwd + bwd}


# ---- from the definitions, in 64 bits

def _exact_steps(q, k, v, g, beta, S, scale):
    o = []
    for t in range(v.shape[1]):
        S, e = _token(k, v, g, beta, S, t)
        o.append(scale * (S * q[:, t, :, :, None]).sum(-2))
    return torch.stack(o, 1), S


def _token(k, v, g, beta, S, t):
    D = S * g[:, t, :, None, None].exp()
    e = v[:, t] - (D * k[:, t, :, :, None]).sum(-2)
    return torch.addcmul(D, k[:, t, :, :, None], (beta[:, t, :, None] * e)[..., None, :]), e


def _exact_rule(q, k, v, g, beta, S0, scale, dO, dS):
    """Token by token, and the adjoint of every token from the last to the first; states are kept at every 64th token."""
    T, S, kept, o = v.shape[1], S0, [], []
    for t in range(T):
        if t % 64 == 0:
            kept.append(S)
        S, _ = _token(k, v, g, beta, S, t)
        o.append(scale * (S * q[:, t, :, :, None]).sum(-2))
    out = {"o": torch.stack(o, 1), "S": S}
    if dO is None:
        return out
    grads = {x: [None] * T for x in ("dq", "dk", "dv", "dg", "dbeta")}
    D = torch.zeros_like(S) if dS is None else dS
    for t0 in range((T - 1) // 64 * 64, -1, -64):
        S, states, errs = kept.pop(), [], []
        for t in range(t0, min(t0 + 64, T)):
            states.append(S)
            S, e = _token(k, v, g, beta, S, t)
            errs.append(e)
        states.append(S)
        for t in range(min(t0 + 64, T) - 1, t0 - 1, -1):
            before, after, e = states[t - t0], states[t - t0 + 1], errs[t - t0]
            kt, bt, a = k[:, t], beta[:, t, :, None], g[:, t, :, None, None].exp()
            grads["dq"][t] = scale * (after * dO[:, t, :, None, :]).sum(-1)
            D = torch.addcmul(D, scale * q[:, t, :, :, None], dO[:, t, :, None, :])
            Dk = (D * kt[..., None]).sum(-2)                                 # adjoint of beta e
            grads["dbeta"][t] = (e * Dk).sum(-1)
            de = bt * Dk
            grads["dv"][t] = de
            decayed = a * before
            grads["dk"][t] = (D * (bt * e)[..., None, :]).sum(-1) - (decayed * de[..., None, :]).sum(-1)
            D = torch.addcmul(D, kt[..., None], de[..., None, :], value=-1.0)
            grads["dg"][t] = (D * decayed).sum((-1, -2))
            D = a * D
    out.update((x, torch.stack(y, 1)) for x, y in grads.items())
    out["dS0"] = D
    return out


def _exact_kept_values(x):
    x = x.double()
    b = x.reshape(*x.shape[:-1], -1, 32)
    mantissa, exponent = torch.frexp(b.abs().amax(-1, keepdim=True))     # a mantissa in [0.5, 1)
    e = torch.where(mantissa > 0, exponent - 1, torch.full_like(exponent, -120)).long()
    step = ((torch.clamp(e, min=-120) + (1023 - 6)) << 52).view(torch.float64)
    return torch.clamp(torch.round(b / step), -127, 127).mul(step).reshape(x.shape)


def _exact_layer(s):
    t = {k: s[k].double() for k in ("x_q", "x_k", "x_v", "o", "g", "dy", "dq", "dk", "dv", "d", "w")}

    def front(x, d):
        q, k, v = (torch.nn.functional.silu(y) for y in x)
        q = q - d[:, None] * k
        return [y / ((y * y).sum(-1, keepdim=True) + EPS).sqrt() for y in (q, k)] + [v]

    def back(o, g, w):
        return torch.sigmoid(g) * w * o / ((o * o).mean(-1, keepdim=True) + EPS).sqrt()

    out = dict(zip("qkv", front([t["x_q"], t["x_k"], t["x_v"]], t["d"])))
    out["y"] = back(t["o"], t["g"], t["w"])
    with torch.enable_grad():
        o, g, w = (x.requires_grad_() for x in (_exact_kept_values(s["o"]), _exact_kept_values(s["g"]), t["w"]))
        out["do"], out["dg"], dw = torch.autograd.grad(back(o, g, w), (o, g, w), t["dy"])
        x = [_exact_kept_values(s[n]).requires_grad_() for n in ("x_q", "x_k", "x_v")]
        d = t["d"].requires_grad_()
        again = front(x, d)
        dxs = torch.autograd.grad(again, (*x, d), [t["dq"], t["dk"], t["dv"]])
    out.update((n + "_again", y.detach()) for n, y in zip("qkv", again))
    out["dx_q"], out["dx_k"], out["dx_v"] = dxs[:3]
    return {**out, "dw": dw, "dd": dxs[3]}


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "kept":
        return _exact_layer(s)
    cu = s.get("cu")
    x = {n: _rows(s[n].double(), cu) for n in ("q", "k", "v", "g", "beta")}
    shared = x["v"].shape[2] // x["q"].shape[2]
    q, k = (x[n].repeat_interleave(shared, 2) for n in "qk")
    if s["kind"] == "step":
        o, S = _exact_steps(q, k, x["v"], x["g"], x["beta"], s["S"].double(), s["scale"])
        return {"o": o, "S": S}
    B, T, H, dv = x["v"].shape
    S0 = torch.zeros(B, H, q.shape[-1], dv, device=q.device, dtype=q.dtype) if s["S0"] is None else s["S0"].double()
    train = s["kind"] == "train"
    r = _exact_rule(q, k, x["v"], x["g"], x["beta"], S0, s["scale"], _rows(s["dO"].double(), cu) if train else None,
                    s["dS"].double() if train and s["segment"] else None)
    for n in ("dq", "dk") if train else ():
        r[n] = r[n].reshape(B, T, H // shared, shared, -1).sum(3)
    out = {n: _packed(r[n], cu) for n in ("o",) + (("dq", "dk", "dv", "dg", "dbeta") if train else ())}
    if not train or s["segment"]:
        out["S"] = r["S"]
    if train and s["segment"]:
        out["dS0"] = r["dS0"]
    return out
