"""Float64 reference of the token operators, each in its defining form (NumPy, no blocking, no chunks)."""
from __future__ import annotations

import numpy as np
from scipy.special import expit, ndtr

ACTIVATIONS = {
    "none": lambda v: v,
    "lrelu": lambda v: np.where(v >= 0, v, 0.1 * v),
    "wsilu": lambda v: v * expit(4 * v),
    "silu": lambda v: v * expit(v),
    "gelu": lambda v: v * ndtr(v),
}


def linear(x, w, b=None, r=None, act="none", gated=False):
    """act(x W^T + b) + r; gated, W = [W1; W2]: act(x W1^T + b1) * (x W2^T + b2) + r."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if b is not None:
        z = z + np.asarray(b, np.float64)
    if gated:
        n = z.shape[-1] // 2
        y = ACTIVATIONS[act](z[..., :n]) * z[..., n:]
    else:
        y = ACTIVATIONS[act](z)
    return y if r is None else y + np.asarray(r, np.float64)


def norm_rope(x, w=None, pos=None, freq=None, sections=(), eps=1e-6, norm=True, interleaved=False):
    """RMS norm of every head of x (tokens, heads, dim), then each pair turned by its axis' position times its frequency."""
    y = np.array(x, np.float64)
    if norm:
        y /= np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        if w is not None:
            y *= np.asarray(w, np.float64)
    P = sum(sections)
    out = y.copy()
    p = 0
    for axis, count in enumerate(sections):
        for _ in range(count):
            angle = np.asarray(pos)[:, axis].astype(np.float64) * float(freq[p])
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
            i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + P)
            out[..., i] = y[..., i] * c - y[..., j] * s
            out[..., j] = y[..., i] * s + y[..., j] * c
            p += 1
    return out


def decay_attention(q, k, v, log_decay, state=None, lengths=None, scale=1.0):
    """S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t S_t, token by token; returns (o, S).

    q (B, T, H, D), k (B, T, K, D), v (B, T, K, V); head h reads key head h // (H // K)."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    B, T, H, D = q.shape
    K, V = k.shape[2], v.shape[3]
    S = np.zeros((B, H, D, V)) if state is None else np.array(state, np.float64)
    o = np.zeros((B, T, H, V))
    lam = np.exp(np.minimum(np.asarray(log_decay, np.float64), 0.0))[:, None, None]
    group = np.arange(H) // (H // K)
    for b in range(B):
        n = T if lengths is None else int(np.clip(lengths[b], 0, T))
        for t in range(n):
            S[b] = lam * S[b] + k[b, t, group][:, :, None] * v[b, t, group][:, None, :]
            o[b, t] = scale * np.einsum("hd,hdv->hv", q[b, t], S[b])
    return o, S
