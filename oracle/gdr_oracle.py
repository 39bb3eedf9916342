"""Oracle of the gated delta rule: fp64, token by token, forward and adjoint, on numpy arrays.

    e_t = v_t - a_t S_{t-1}^T k_t,   S_t = a_t S_{t-1} + beta_t k_t e_t^T,   o_t = scale S_t^T q_t,   a_t = exp(g_t)

q, k [B, T, Hk, dk], v [B, T, H, dv], g, beta [B, T, H], states [B, H, dk, dv]; value head h reads key head h // (H / Hk).
"""
import numpy as np


def _heads(x, H):
    return np.repeat(x, H // x.shape[2], axis=2)


def forward(q, k, v, g, beta, S0=None, scale=1.0, keep=False):
    """dict(o, S, e); keep: also the states after every token, [T + 1][B, H, dk, dv]."""
    B, T, H, dv = v.shape
    q, k, a = _heads(q, H), _heads(k, H), np.exp(g)
    S = np.zeros((B, H, q.shape[-1], dv)) if S0 is None else S0.astype(np.float64).copy()
    o, e, states = np.empty_like(v), np.empty_like(v), [S]
    for t in range(T):
        D = a[:, t, :, None, None] * S
        e[:, t] = v[:, t] - np.einsum("bhk,bhkv->bhv", k[:, t], D)
        S = D + np.einsum("bhk,bhv->bhkv", beta[:, t, :, None] * k[:, t], e[:, t])
        o[:, t] = scale * np.einsum("bhk,bhkv->bhv", q[:, t], S)
        states.append(S)
    return {"o": o, "S": S, "e": e, **({"states": states} if keep else {})}


def backward(q, k, v, g, beta, dO, S0=None, dS=None, scale=1.0):
    """Adjoint of <o, dO> + <S_T, dS>: dict(dq, dk, dv, dg, dbeta, dS0)."""
    B, T, H, dv = v.shape
    Hk, dkn = q.shape[2], q.shape[-1]
    f = forward(q, k, v, g, beta, S0, scale, keep=True)
    qh, kh, a = _heads(q, H), _heads(k, H), np.exp(g)
    D = np.zeros((B, H, dkn, dv)) if dS is None else dS.astype(np.float64).copy()
    dq, dk = np.zeros((B, T, H, dkn)), np.zeros((B, T, H, dkn))
    dvv, dg, dbeta = np.zeros_like(v), np.zeros_like(g), np.zeros_like(g)
    for t in range(T - 1, -1, -1):
        S, e = f["states"][t + 1], f["e"][:, t]
        decayed = a[:, t, :, None, None] * f["states"][t]
        dq[:, t] = scale * np.einsum("bhkv,bhv->bhk", S, dO[:, t])
        D = D + scale * np.einsum("bhk,bhv->bhkv", qh[:, t], dO[:, t])
        De = np.einsum("bhkv,bhv->bhk", D, e)
        Dk = np.einsum("bhkv,bhk->bhv", D, kh[:, t])
        dbeta[:, t] = np.einsum("bhk,bhk->bh", De, kh[:, t])
        de = beta[:, t, :, None] * Dk
        dvv[:, t] = de
        dk[:, t] = beta[:, t, :, None] * De - np.einsum("bhkv,bhv->bhk", decayed, de)
        D = D - np.einsum("bhk,bhv->bhkv", kh[:, t], de)
        dg[:, t] = np.einsum("bhkv,bhkv->bh", D, decayed)
        D = a[:, t, :, None, None] * D
    fold = lambda x: x.reshape(B, T, Hk, H // Hk, dkn).sum(3)
    return {"dq": fold(dq), "dk": fold(dk), "dv": dvv, "dg": dg, "dbeta": dbeta, "dS0": D}
