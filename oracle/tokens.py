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


def seen(i, window=None, sinks=0):
    """The tokens that token i sees: j <= i with i - j < window (None: all) or j < sinks."""
    j = np.arange(i + 1)
    return j if window is None else j[(i - j < window) | (j < sinks)]


def _softmax_rows(z):
    e = np.exp(z - z.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def window_attention(q, k, v, window=None, sinks=0, lengths=None, scale=1.0):
    """Softmax attention of every token over the tokens that it sees; q (B, T, H, D), k (B, T, K, D), v (B, T, K, V)."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    B, T, H, _ = q.shape
    K, V = k.shape[2], v.shape[3]
    o = np.zeros((B, T, H, V))
    head = np.arange(H) // (H // K)
    for b in range(B):
        n = T if lengths is None else int(np.clip(lengths[b], 0, T))
        for i in range(n):
            j = seen(i, window, sinks)
            p = _softmax_rows(scale * np.matmul(k[b, j].transpose(1, 0, 2)[head], q[b, i, :, :, None])[..., 0])
            o[b, i] = np.matmul(p[:, None], v[b, j].transpose(1, 0, 2)[head])[:, 0]
    return o


def _positions(table, pages, page, n):
    """(position, page, row) of the first n positions that have a page."""
    j = np.arange(n)
    p = np.asarray(table)[j // page].astype(np.int64) if n else j
    ok = (p >= 0) & (p < pages)
    return j[ok], p[ok], j[ok] % page


def paged_attention(q, k_cache, v_cache, table, lengths, window=None, sinks=0, scale=1.0, mass=None):
    """The last token of each sequence over its cache; q (B, H, D), caches (pages, page, K, .); returns (o, mass)."""
    q, kc, vc = (np.asarray(a, np.float64) for a in (q, k_cache, v_cache))
    B, H, _ = q.shape
    pages, page, K, V = vc.shape
    o = np.zeros((B, H, V))
    mass = None if mass is None else np.array(mass, np.float64)
    for b in range(B):
        n = int(np.clip(lengths[b], 0, page * np.shape(table)[1]))
        j, p, r = _positions(table[b], pages, page, n)
        ok = np.isin(j, seen(n - 1, window, sinks))
        j, p, r = j[ok], p[ok], r[ok]
        if not len(j):
            continue
        for h in range(H):
            w = _softmax_rows(scale * (kc[p, r, h // (H // K)] @ q[b, h]))
            o[b, h] = w @ vc[p, r, h // (H // K)]
            if mass is not None:
                mass[b, h // (H // K), j] += w
    return o, mass


def cache_append(k, v, k_cache, v_cache, table, starts, counts=None, mass=None):
    """Token i of sequence b to position starts[b] + i; returns the new (k_cache, v_cache, mass)."""
    kc, vc = np.array(k_cache), np.array(v_cache)
    mass = None if mass is None else np.array(mass)
    pages, page = kc.shape[:2]
    B, T = np.shape(k)[:2]
    for b in range(B):
        n = T if counts is None else int(np.clip(counts[b], 0, T))
        for i in range(n):
            j = int(starts[b]) + i
            if not 0 <= j < page * np.shape(table)[1] or not 0 <= table[b][j // page] < pages:
                continue
            kc[table[b][j // page], j % page] = k[b][i]
            vc[table[b][j // page], j % page] = v[b][i]
            if mass is not None:
                mass[b, :, j] = 0
    return kc, vc, mass


def cache_evict(k_cache, v_cache, table, lengths, mass, keep, new_table, sinks=0, recent=0):
    """The heaviest tokens of each sequence and key head to new pages; returns (k_cache, v_cache, lengths, mass, kept)."""
    kc, vc, mass = np.array(k_cache), np.array(v_cache), np.asarray(mass)
    pages, page, K = kc.shape[:3]
    B = len(lengths)
    new_lengths = np.zeros(B, np.int32)
    new_mass = np.zeros((B, K, page * np.shape(new_table)[1]), np.float32)
    kept = np.full((B, K, keep), -1, np.int32)
    for b in range(B):
        n = int(np.clip(lengths[b], 0, page * np.shape(table)[1]))
        new_lengths[b] = m = min(n, keep)
        for h in range(K):
            # fixed ones first, then NaN, then by weight, then by position
            key = lambda j: (not (j < sinks or j >= n - recent), not np.isnan(mass[b, h, j]),  # noqa: E731
                             0.0 if np.isnan(mass[b, h, j]) else -mass[b, h, j], j)
            got = sorted(sorted(range(n), key=key)[:m])
            kept[b, h, :m] = got
            new_mass[b, h, :m] = mass[b, h, got]
            for x, j in enumerate(got):
                src, dst = table[b][j // page], new_table[b][x // page]
                if 0 <= src < pages and 0 <= dst < pages:
                    kc[dst, x % page, h] = k_cache[src, j % page, h]
                    vc[dst, x % page, h] = v_cache[src, j % page, h]
    return kc, vc, new_lengths, new_mass, kept
