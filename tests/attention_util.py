"""Shared by the tests of the attentions over latent tokens: inputs, caches, and how far outputs may be off.

Of a score, fp32: (D + 2) products and sums against the sum of magnitudes, and four more operations on its value.  A
weight then errs by that, by 2^-21 of the exponential, and by its two 16-bit terms (2^-22 in fp16, 2^-16 in bf16, and in
fp16 2^-32 of the largest weight where the terms are subnormal).  Weights occur above and below the line, their sums are
fp32; the output is rounded once."""
import numpy as np
import torch

from oracle import tokens as ref

DEV = "cuda:0"
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
U = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -133}
F32 = 2.0 ** -24


def say(*a):
    print("[gpu-attention]", *a, flush=True)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rnd(g, shape, dt, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(DT[dt])


def f64(t):
    return t.detach().cpu().double().numpy()


def weight_error(q, k, scale, D, dt):
    """Relative error of a weight against its formula, over all pairs (their largest magnitudes)."""
    mag = abs(scale) * np.abs(q).max() * np.abs(k).max() * D if q.size and k.size else 0.0
    return (D + 6) * F32 * mag + 2.0 ** -21 + (2.0 ** -22 if dt == "fp16" else 2.0 ** -16)


def output_bound(want, mag, vmax, q, k, scale, D, n, dt):
    """want: the outputs, mag: the same weights over magnitudes of v, n: tokens seen at most."""
    e = (2 * weight_error(q, k, scale, D, dt) + (n + 64) * F32) * mag
    if dt == "fp16":
        e = e + n * 2.0 ** -32 * vmax
    return e * (1 + U[dt]) + U[dt] * np.abs(want) + TINY[dt]


def check(got, want, bound, what):
    got = f64(got)
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), (what, float(over.max()), np.unravel_index(over.argmax(), over.shape))


def check_rounding(got, want, dt, what):
    """Nothing but the last rounding counts: it is at most U, uniform, so its rms at most U / sqrt(3) = 0.578 U."""
    norm = np.sqrt((want ** 2).mean())
    if norm:
        assert np.sqrt(((f64(got) - want) ** 2).mean()) <= 0.6 * U[dt] * norm, what


def sequences(g, B, T, heads, d, dt, layout="packed", offset=0, pad=0, scale=1.0):
    """(B, T, heads, d) views on the GPU: tokens or heads next to each other, rows padded, the first element offset."""
    shape = (B, heads, T, d + pad) if layout == "heads" else (B, T, heads, d + pad)
    n = int(np.prod(shape))
    buf = rnd(g, (n + offset,), dt, scale).to(DEV)[offset:].view(shape)[..., :d]
    return buf.transpose(1, 2) if layout == "heads" else buf


class Cache:
    """A cache with pages in no order; layout: pages of tokens, of heads, or keys and values side by side in a page."""

    def __init__(self, g, B, capacity, page, K, D, V, dt, layout="tokens", spare=2, extra_columns=0, fill=1.0):
        per = -(-capacity // page)
        self.pages, self.page, self.K, self.D, self.V, self.dt = B * per + spare, page, K, D, V, dt
        if layout == "heads":
            self.k = rnd(g, (self.pages, K, page, D), dt, fill).to(DEV).transpose(1, 2)
            self.v = rnd(g, (self.pages, K, page, V), dt, fill).to(DEV).transpose(1, 2)
        elif layout == "beside":
            kv = rnd(g, (self.pages, page, K, D + V), dt, fill).to(DEV)
            self.k, self.v = kv[..., :D], kv[..., D:]
        else:
            self.k, self.v = rnd(g, (self.pages, page, K, D), dt, fill).to(DEV), rnd(g, (self.pages, page, K, V), dt, fill).to(DEV)
        ids = torch.randperm(self.pages, generator=g)
        table = ids[:B * per].reshape(B, per).to(torch.int32)
        wide = torch.full((B, per + extra_columns), -7, dtype=torch.int32)
        wide[:, :per] = table
        self.free = ids[B * per:]
        self.table = wide.to(DEV)[:, :per] if extra_columns else table.to(DEV)
        self.columns = per * page


def paged_reference(q, c, lengths, window, sinks, scale, mass=None, table=None):
    args = (f64(c.table if table is None else table).astype(np.int64), f64(lengths).astype(np.int64), window, sinks, scale)
    want, wm = ref.paged_attention(f64(q), f64(c.k), f64(c.v), *args, None if mass is None else f64(mass))
    mag, _ = ref.paged_attention(f64(q), f64(c.k), np.abs(f64(c.v)), *args)
    return want, mag, wm
