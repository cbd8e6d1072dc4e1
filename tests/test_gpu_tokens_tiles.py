"""The large kernels of the token operators: every tile of the matrix product and every form of the chunked attention,
at sizes that the rules send to them (``test_tokens_rules.py`` holds the lists to that), against 64 bits on the GPU.

Bounds are those of ``test_gpu_tokens.py`` and ``test_gpu_tokens_bounds.py``."""
import numpy as np
import pytest
import torch

from oracle import tokens as ref
from paper_2502_20762_amd import tokens as tk
from test_gpu_tokens import DEV, DT, F32, TINY, U, f64, gen, rnd, say
from test_gpu_tokens_bounds import TERMS

pytestmark = pytest.mark.gpu

ACTS = ("none", "lrelu", "wsilu", "silu", "gelu")

# kernel: (rows, k, weight rows, padding of x's rows); remainders of every tile, contractions below a stage, of one, with a tail
LINEAR = {
    "rows16": [(9, 1200, 1030, 0), (90, 264, 1000, 8)],
    "rows32": [(27, 520, 6000, 0), (150, 65, 1200, 3)],
    "rows64": [(500, 136, 1030, 0), (1001, 72, 500, 0)],
    "reg128x64": [(1001, 77, 778, 0), (700, 264, 1030, 1), (513, 5, 1100, 0)],
    "reg128x128": [(8001, 77, 778, 3), (8001, 33, 900, 0)],
    "reg256x256": [(9700, 130, 1100, 0), (9473, 40, 1026, 1)],
    "dma128x64": [(1001, 72, 778, 0), (700, 512, 1030, 8), (520, 8, 1100, 0), (1001, 1096, 1034, 0)],
    "dma128x128": [(8001, 72, 778, 0), (8100, 264, 900, 8), (7950, 8, 770, 0), (8001, 504, 778, 0)],
    "dma256x128k32": [(16400, 72, 2050, 0), (16300, 264, 2050, 8), (16400, 8, 2060, 0), (16131, 512, 2300, 0)],
    "dma256x128k64": [(4100, 520, 1290, 0), (3900, 1096, 1300, 8), (8160, 512, 1000, 0)],
    "dma256x256": [(8300, 520, 1290, 0), (8200, 1096, 1300, 8), (8321, 512, 1290, 0)],
}


def plain(x, w, b, r, act, gated):
    """The product in float64 on the GPU, and the bound of its error (as ``linear_bound`` has it)."""
    def activation(v):
        return {"none": lambda: v, "lrelu": lambda: torch.where(v >= 0, v, 0.1 * v), "wsilu": lambda: v * torch.sigmoid(4 * v),
                "silu": lambda: v * torch.sigmoid(v), "gelu": lambda: v * torch.special.ndtr(v)}[act]()

    x, w = x.double(), w.double()
    wt = w.t().contiguous()
    z, mag = x @ wt, x.abs() @ wt.abs()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    e = (x.shape[1] + 4) * F32 * mag
    if gated:
        n = w.shape[0] // 2
        a = activation(z[:, :n])
        y = a * z[:, n:]
        a = a.abs()
        e = (1.13 * e[:, :n] + 2.0 ** -19 * a) * (z[:, n:].abs() + e[:, n:]) + a * e[:, n:]
    else:
        y = activation(z)
        e = 1.13 * e + 2.0 ** -19 * y.abs()
    rd = 0 if r is None else r.double()
    y = y + rd
    e = e + 4 * F32 * (y.abs() + (0 if r is None else rd.abs()))
    return y, e


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kernel", list(LINEAR))
def test_every_kernel_of_the_product(kernel, gated, dt):
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(map(ord, kernel)))

    def made(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(DT[dt])

    runs = [(LINEAR[kernel][i % len(LINEAR[kernel])], act, i) for i, act in enumerate(ACTS)]
    for (m, k, rows, pad), act, i in runs:
        say(kernel, gated, dt, m, k, rows, act)
        n = rows // 2 if gated else rows
        x, w = made(m, k + pad)[:, :k], made(rows, k, scale=k ** -0.5)
        b = made(rows) if i != 1 else None
        r = made(m, n + pad)[:, :n] if i % 2 == 0 else None
        y, e = plain(x, w, b, r, act, gated)
        buf = torch.full((m + 1, n + 3), 7.0, dtype=DT[dt], device=DEV)  # rows of an odd width, one more behind them
        out = buf[:m, :n]
        tk.linear(x, w, b, residual=r, act=act, gated=gated, out=out)
        bound = e * (1 + U[dt]) + U[dt] * y.abs() + TINY[dt]
        over = (out.double() - y).abs() - bound
        assert bool(torch.isfinite(out).all()) and float(over.max()) <= 0, (m, k, rows, act, float(over.max()))
        assert bool((buf[:, n:] == 7.0).all()) and bool((buf[m] == 7.0).all())
        if r is not None:  # in place of the residual, and again: the same values
            want = out.contiguous()
            same = tk.linear(x, w, b, residual=r, act=act, gated=gated)
            tk.linear(x, w, b, residual=r, act=act, gated=gated, out=r)
            assert torch.equal(same, want) and torch.equal(r, want)


@pytest.mark.parametrize("kernel", [k for k in LINEAR if "x" in k])
def test_nan_and_infinities_stay_in_their_rows_in_every_tile(kernel):
    m, k, rows, pad = LINEAR[kernel][0]
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    x = torch.randn((m, k + pad), generator=g, device=DEV).half()[:, :k]
    w = (torch.randn((rows, k), generator=g, device=DEV) * k ** -0.5).half()
    clean = tk.linear(x, w, act="gelu")
    x[1, 3], x[m - 1, k - 1], x[m // 2, 0] = float("inf"), float("nan"), float("nan")
    y = tk.linear(x, w, act="gelu")
    ok = torch.ones(m, dtype=torch.bool, device=DEV)
    ok[1] = ok[m - 1] = ok[m // 2] = False
    assert torch.equal(y[ok], clean[ok])
    assert bool(torch.isnan(y[m - 1]).all()) and bool(torch.isnan(y[m // 2]).all()) and not bool(torch.isfinite(y[1]).all())


# ---------------------------------------------------------------- attention with a decay
# what the case is for: (batch, tokens, heads, key heads, head_dim, value_dim, lengths)
DECAY = {
    "one segment of 18 chunks": (1, 1100, 256, 128, 8, 128, None),
    "one segment of 18 chunks, wide": (1, 1100, 256, 256, 72, 65, None),
    "one segment, narrow values": (8, 1160, 128, 32, 16, 24, [1160, 0, 1, 1023, 1024, 1025, 1088, 700]),
    "two segments of 19 chunks": (1, 2400, 255, 255, 8, 128, None),
    "segments of 17 chunks, odd": (1, 2160, 255, 51, 9, 67, [2159]),
    "67 segments": (7, 8570, 1, 1, 32, 32, [8570, 8064, 8065, 8192, 8193, 8321, 8449]),
    "67 segments, odd": (1, 8570, 1, 1, 33, 31, None),
    "209 segments": (1, 40000, 1, 1, 64, 16, None),
    "157 segments, wide": (1, 20050, 2, 1, 128, 128, None),
    "odd state of many segments": (2, 700, 3, 1, 75, 33, [700, 470]),
}
FORMS = [(D, V) for D in (24, 64, 72, 128) for V in (16, 32, 40, 64, 72, 128)] + [(D, V) for D in (33, 127) for V in (31, 50, 127)]


def recurrence(q, k, v, ld, S, lengths, scale):
    """Token by token in float64 on the GPU; (o, S)."""
    q, k, v, S = (t.double() for t in (q, k, v, S))
    B, T, H, _ = q.shape
    rep = H // k.shape[2]
    k, v = (t.repeat_interleave(rep, 2) for t in (k, v))
    lam = torch.exp(ld.double().clamp(max=0))[:, None, None]
    n = torch.full((B,), T, device=DEV) if lengths is None else lengths
    o = torch.zeros((B, T, H, v.shape[-1]), dtype=torch.float64, device=DEV)
    for t in range(T):
        new = torch.addcmul(S * lam, k[:, t, :, :, None], v[:, t, :, None, :])
        live = (t < n)[:, None, None]
        S = torch.where(live[..., None], new, S) if lengths is not None else new
        o[:, t] = torch.where(live, scale * (q[:, t, :, :, None] * S).sum(2), 0.0)
    return o, S


def attend(B, T, H, K, D, V, lengths, dt, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def made(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(DT[dt])

    q, k, v = made(B, T, H, D), made(B, T, K, D), made(B, T, K, V)
    ld = -torch.tensor([0.3, 0.02, 0.0005, 0.0], device=DEV).repeat(-(-H // 4))[:H].contiguous()
    S0 = torch.randn((B, H, D, V), generator=g, device=DEV) * 3
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    if ln is not None:  # past a sequence's end nothing is read
        for b, n in enumerate(lengths):
            q[b, n:], k[b, n:], v[b, n:] = float("nan"), float("inf"), float("nan")
    scale = D ** -0.5
    o, S = tk.decay_attention(q, k, v, ld, S0, ln, scale, return_state=True)
    if ln is not None:
        for b, n in enumerate(lengths):
            q[b, n:], k[b, n:], v[b, n:] = 0.0, 0.0, 0.0
    want, wS = recurrence(q, k, v, ld, S0, ln, scale)
    mag, mS = recurrence(q.abs(), k.abs(), v.abs(), ld, S0.abs(), ln, scale)
    # a chunk's sums and 64 at most of its terms and the segments before it, however long the sequence is: each step of the
    # state rounds what was there (T of them) only where nothing decays
    e = (TERMS[dt] + (T + 256) * F32) * mag
    over = (o.double() - want).abs() - (e * (1 + U[dt]) + U[dt] * want.abs() + TINY[dt])
    assert bool(torch.isfinite(o).all()) and float(over.max()) <= 0, float(over.max())
    over = (S.double() - wS).abs() - (((T + 16) * F32 + 2.0 ** -21) * mS + 1e-37)
    assert bool(torch.isfinite(S).all()) and float(over.max()) <= 0, ("state", float(over.max()))
    # over all elements the error is that of the rounding, and of the fp32 state
    rounded = want.to(DT[dt]).double()
    assert ((o.double() - want) ** 2).mean() <= 1.05 ** 2 * ((rounded - want) ** 2).mean()
    assert ((S.double() - wS) ** 2).mean() <= (2.0 ** -18) ** 2 * (wS ** 2).mean()
    if ln is not None:
        for b, n in enumerate(lengths):
            assert bool((o[b, n:] == 0).all())


def test_the_recurrence_is_the_oracles():
    g = gen(8)
    q, k, v = rnd(g, (2, 20, 4, 16), "fp16"), rnd(g, (2, 20, 2, 16), "fp16"), rnd(g, (2, 20, 2, 24), "fp16")
    ld, S0 = torch.tensor([-0.1, 0.0, -0.5, -3.0]), torch.randn((2, 4, 16, 24), generator=g)
    ln = torch.tensor([20, 7], dtype=torch.int32)
    o, S = recurrence(*(t.to(DEV) for t in (q, k, v, ld, S0, ln)), 0.25)
    want, wS = ref.decay_attention(*(f64(t) for t in (q, k, v, ld, S0)), [20, 7], 0.25)
    assert np.abs(f64(o) - want).max() <= 1e-12 * np.abs(want).max() and np.abs(f64(S) - wS).max() <= 1e-12 * np.abs(wS).max()


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("case", list(DECAY))
def test_long_sequences(case, dt):
    say("decay", case, dt)
    attend(*DECAY[case], dt, 3)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("D,V", FORMS)
def test_every_width_in_segments(D, V, dt):
    say("decay in segments", D, V, dt)
    attend(2, 400, 2, 1, D, V, [400, 333], dt, 4)
