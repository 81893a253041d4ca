"""Float64 oracle of the layers: linear attention with a decay for each head (step by step, and its
reverse mode written from the recurrence) and layer normalisation."""
from __future__ import annotations

import numpy as np

f64 = np.float64


def _lengths(lengths, B, T):
    return np.full(B, T) if lengths is None else np.clip(np.asarray(lengths, np.int64), 0, T)


def _operands(q, k, v, log_decay):
    """float64 operands with shared q, k heads repeated, decays [B, T, H]."""
    q, k, v = (np.asarray(x, f64) for x in (q, k, v))
    B, T, H, _ = v.shape
    r = H // q.shape[2]
    a = np.exp(np.broadcast_to(np.asarray(log_decay, f64), (B, T, H)))
    return np.repeat(q, r, 2), np.repeat(k, r, 2), v, a, r


def linattn(q, k, v, log_decay, scale=1.0, lengths=None, state0=None):
    """o [B,T,H,Dv] and the last state [B,H,Dk,Dv]: S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t."""
    q, k, v, a, _ = _operands(q, k, v, log_decay)
    B, T, H, Dv = v.shape
    n = _lengths(lengths, B, T)
    o = np.zeros((B, T, H, Dv), f64)
    last = np.zeros((B, H, k.shape[3], Dv), f64) if state0 is None else np.array(state0, f64)
    for b in range(B):
        S = last[b]
        for t in range(n[b]):
            S = a[b, t, :, None, None] * S + k[b, t, :, :, None] * v[b, t, :, None, :]
            o[b, t] = scale * np.einsum("hd,hdn->hn", q[b, t], S)
        last[b] = S
    return o, last


def linattn_adjoint(q, k, v, log_decay, g, scale=1.0, lengths=None, state0=None, g_state=None):
    """dict(q, k, v, log_decay, state0): gradients of <o, g> + <last state, g_state>; log_decay of the
    given shape."""
    ld = np.asarray(log_decay, f64)
    q, k, v, a, r = _operands(q, k, v, ld)
    g = np.asarray(g, f64)
    B, T, H, Dv = v.shape
    Dk = k.shape[3]
    n = _lengths(lengths, B, T)
    dq, dk, dv, da = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros((B, T, H), f64)
    ds0 = np.zeros((B, H, Dk, Dv), f64)
    for b in range(B):
        S = [np.zeros((H, Dk, Dv), f64) if state0 is None else np.asarray(state0[b], f64)]
        for t in range(n[b]):
            S.append(a[b, t, :, None, None] * S[-1] + k[b, t, :, :, None] * v[b, t, :, None, :])
        R = np.zeros((H, Dk, Dv), f64) if g_state is None else np.asarray(g_state[b], f64)
        for t in range(n[b] - 1, -1, -1):
            R = R + scale * q[b, t, :, :, None] * g[b, t, :, None, :]
            dq[b, t] = scale * np.einsum("hdn,hn->hd", S[t + 1], g[b, t])
            dk[b, t] = np.einsum("hdn,hn->hd", R, v[b, t])
            dv[b, t] = np.einsum("hdn,hd->hn", R, k[b, t])
            R = a[b, t, :, None, None] * R
            da[b, t] = np.einsum("hdn,hdn->h", R, S[t])
        ds0[b] = R
    Hk = H // r
    return {"q": dq.reshape(B, T, Hk, r, Dk).sum(3), "k": dk.reshape(B, T, Hk, r, Dk).sum(3), "v": dv,
            "log_decay": da if ld.ndim == 3 else da.sum((0, 1)), "state0": ds0}


def layernorm(x, w=None, b=None, eps=1e-5):
    """(y, mean, rstd) over the last axis."""
    x = np.asarray(x, f64)
    mean = x.mean(-1)
    d = x - mean[..., None]
    rstd = 1.0 / np.sqrt((d * d).mean(-1) + eps)
    y = d * rstd[..., None]
    if w is not None:
        y = y * np.asarray(w, f64)
    if b is not None:
        y = y + np.asarray(b, f64)
    return y, mean, rstd


def layernorm_adjoint(x, g, w=None, eps=1e-5, groups=False):
    """dict(x, w, b) for the cotangent g of y; groups: weights [G, D] for x [..., G, D]."""
    x, g = np.asarray(x, f64), np.asarray(g, f64)
    _, mean, rstd = layernorm(x, eps=eps)
    xh = (x - mean[..., None]) * rstd[..., None]
    u = g if w is None else g * np.asarray(w, f64)
    dx = rstd[..., None] * (u - u.mean(-1, keepdims=True) - xh * (u * xh).mean(-1, keepdims=True))
    tail = x.shape[-2:] if groups else x.shape[-1:]
    return {"x": dx, "w": (g * xh).reshape(-1, *tail).sum(0), "b": g.reshape(-1, *tail).sum(0)}
