"""Token operators on the GPU against the float64 oracle.

Bounds are element by element, from the formats: u is the unit roundoff of the output type (2^-11 fp16, 2^-8 bf16),
sums are fp32 (relative 2^-24 an operation, against the sum of magnitudes), and where a kernel rounds an intermediate
to 16 bits, that rounding's worst case against magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import tokens as ref
from paper_2502_20762_amd import ncodec as nc
from paper_2502_20762_amd import tokens as tk

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
U = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -133}
F32 = 2.0 ** -24


def say(*a):
    print("[gpu-tokens]", *a, flush=True)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rnd(g, shape, dt, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(DT[dt])


def f64(t):
    return t.detach().cpu().double().numpy()


def check(got, want, bound, what):
    got = f64(got)
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), (what, float(over.max()), np.unravel_index(over.argmax(), over.shape))


# ---------------------------------------------------------------- linear
def linear_bound(x, w, b, r, act, gated, dt, want):
    """Errors of the fp32 sums through the activation (slope at most 1.13), of the activation, and of the rounding."""
    K = x.shape[1]
    mag = np.abs(x) @ np.abs(w).T + (0 if b is None else np.abs(b))
    e = (K + 4) * F32 * mag
    z = x @ w.T + (0 if b is None else b)
    if gated:
        n = w.shape[0] // 2
        a = np.abs(ref.ACTIVATIONS[act](z[:, :n]))
        e = (1.13 * e[:, :n] + 2.0 ** -19 * a) * (np.abs(z[:, n:]) + e[:, n:]) + a * e[:, n:]
    else:
        e = 1.13 * e + 2.0 ** -19 * np.abs(ref.ACTIVATIONS[act](z))
    e = e + 4 * F32 * (np.abs(want) + (0 if r is None else np.abs(r)))
    return e * (1 + U[dt]) + U[dt] * np.abs(want) + TINY[dt]


def run_linear(m, k, n, dt, act="none", gated=False, bias=True, residual=False, padx=0, padw=0, pady=0, offset=0,
               inplace=False, seed=0):
    g = gen(seed)
    nw = 2 * n if gated else n

    def rows(count, width, pad, scale=1.0):
        buf = rnd(g, (count * (width + pad) + offset,), dt, scale).to(DEV)
        return buf[offset:].view(count, width + pad)[:, :width]

    x, w = rows(m, k, padx), rows(nw, k, padw, k ** -0.5)
    b = rnd(g, (nw,), dt).to(DEV) if bias else None
    r = rows(m, n, pady) if residual else None
    want = ref.linear(f64(x), f64(w), None if b is None else f64(b), None if r is None else f64(r), act, gated)
    bound = linear_bound(f64(x), f64(w), None if b is None else f64(b), None if r is None else f64(r), act, gated, dt,
                         want)
    buf = torch.full((m * (n + pady) + offset + 64,), 7.0, dtype=DT[dt], device=DEV)
    out = r if inplace else buf[offset:offset + m * (n + pady)].view(m, n + pady)[:, :n]
    got = tk.linear(x, w, b, residual=r, act=act, gated=gated, out=out)
    torch.cuda.synchronize()
    check(got, want, bound, (m, k, n, dt, act, gated))
    if not inplace:  # nothing written around the rows
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep[offset:offset + m * (n + pady)].view(m, n + pady)[:, :n] = False
        assert bool((buf[keep] == 7.0).all())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("m,k,n", [
    (1, 1, 1), (1, 512, 2048), (1, 33, 65), (2, 64, 64), (3, 100, 17), (16, 256, 768), (17, 2048, 48), (31, 72, 129),
    (64, 64, 64), (65, 65, 65), (127, 96, 200), (128, 256, 256), (200, 40, 8), (257, 520, 264), (500, 130, 1030),
    (1560, 128, 384), (700, 1000, 333),
])
def test_linear_sizes(m, k, n, dt):
    say("linear", m, k, n, dt)
    run_linear(m, k, n, dt, residual=(m % 2 == 0))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "lrelu", "wsilu", "silu", "gelu"])
@pytest.mark.parametrize("m,k,n", [(1, 96, 72), (40, 64, 96), (300, 192, 264)])
def test_linear_epilogues(m, k, n, act, gated, dt):
    say("linear", m, k, n, act, gated, dt)
    run_linear(m, k, n, dt, act, gated, bias=True, residual=True)
    run_linear(m, k, n, dt, act, gated, bias=False, residual=False, seed=1)


@pytest.mark.parametrize("m,k,n", [(1, 64, 40), (70, 256, 130), (700, 512, 512), (260, 77, 300)])
@pytest.mark.parametrize("padx,padw,pady,offset", [(8, 8, 8, 0), (1, 3, 5, 0), (0, 0, 0, 1), (3, 0, 1, 3), (8, 0, 4, 4)])
def test_linear_strides_and_alignment(m, k, n, padx, padw, pady, offset):
    say("linear strides", m, k, n, padx, padw, pady, offset)
    for gated in (False, True):
        run_linear(m, k, n, "fp16", "silu", gated, True, True, padx, padw, pady, offset)


@pytest.mark.parametrize("m,n", [(1, 64), (50, 72), (600, 512), (33, 31)])
def test_linear_in_place_residual(m, n):
    run_linear(m, 128, n, "bf16", "gelu", False, True, True, inplace=True)


def test_linear_infinities_and_nan_stay_in_their_rows():
    g = gen(3)
    for m, k, n in ((5, 70, 90), (300, 256, 256)):
        x, w = rnd(g, (m, k), "fp16"), rnd(g, (n, k), "fp16", k ** -0.5)
        clean = tk.linear(x.to(DEV), w.to(DEV), act="silu").cpu()
        x2 = x.clone()
        x2[1, 3], x2[m - 1, k - 1] = float("inf"), float("nan")
        y = tk.linear(x2.to(DEV), w.to(DEV), act="silu").cpu()
        rows = torch.ones(m, dtype=torch.bool)
        rows[1] = rows[m - 1] = False
        assert torch.equal(y[rows], clean[rows])
        assert not torch.isfinite(y[m - 1]).any() and not torch.isfinite(y[1]).all()


def test_linear_saturated_activations():
    # far out, the logistic and erfc end at 0 and 1, never at a NaN
    x = torch.tensor([[-6e4], [-200.0], [-30.0], [0.0], [30.0], [200.0], [6e4]], dtype=torch.float16, device=DEV)
    w = torch.ones((1, 1), dtype=torch.float16, device=DEV)
    for act in ("wsilu", "silu", "gelu", "lrelu"):
        y = f64(tk.linear(x, w, act=act))[:, 0]
        want = ref.ACTIVATIONS[act](f64(x)[:, 0])
        assert np.isfinite(y).all() and np.abs(y - want).max() <= 2.0 ** -11 * np.abs(want).max()
        assert (np.abs(y[:3]) <= np.abs(want[:3]) * 1.001 + 2.0 ** -24).all(), (act, y)


def test_linear_leading_dimensions_and_empty():
    g = gen(4)
    x, w = rnd(g, (2, 3, 5, 64), "fp16").to(DEV), rnd(g, (32, 64), "fp16").to(DEV)
    y = tk.linear(x, w)
    assert y.shape == (2, 3, 5, 32) and torch.equal(y.view(-1, 32), tk.linear(x.view(-1, 64), w))
    assert torch.equal(tk.linear(x[0, 0, 0], w), y[0, 0, 0])
    assert tk.linear(x[:, :0], w).shape == (2, 0, 5, 32)


def test_linear_rows_past_32_bit_offsets():
    ld = (1 << 30) + 24  # rows 2 and 3 begin past 2^31 elements
    buf = torch.empty(3 * ld + 4096, dtype=torch.float16, device=DEV)
    x = buf.as_strided((4, 64), (ld, 1))
    x.copy_(rnd(gen(5), (4, 64), "fp16"))
    w = rnd(gen(6), (40, 64), "fp16").to(DEV)
    assert torch.equal(tk.linear(x, w), tk.linear(x.contiguous(), w))
    y = buf.as_strided((4, 40), (ld, 1), 1024)
    assert torch.equal(tk.linear(x.contiguous(), w, out=y), tk.linear(x.contiguous(), w))


def test_linear_more_rows_than_a_launch_takes():
    m = (1 << 28) + 1000  # one product an output: the rounding of an exact fp32 value
    x = torch.arange(m, device=DEV, dtype=torch.int32).remainder_(1999).to(torch.float16).view(m, 1)
    w = torch.tensor([[0.375]], dtype=torch.float16, device=DEV)
    y = tk.linear(x, w, residual=x)
    for lo in range(0, m, 1 << 26):  # 1.375 x is 11 x / 8: fp32 holds it, fp16 rounds it once
        part = x[lo:lo + (1 << 26)].float()
        assert torch.equal(y[lo:lo + (1 << 26)], (part * 0.375 + part).half()), lo


def test_linear_is_repeatable_and_takes_the_current_stream():
    g = gen(7)
    x, w = rnd(g, (900, 512), "bf16").to(DEV), rnd(g, (300, 512), "bf16").to(DEV)
    a = tk.linear(x, w, act="gelu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = tk.linear(x, w, act="gelu")
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, b)


# ---------------------------------------------------------------- norms and rotation
def rope_bound(x, w, pos, freq, sections, eps, norm, inter, dt, want):
    """fp32 norm (a few operations on a sum of D) and rotation (sine and cosine to 2^-19), then one rounding."""
    D = x.shape[-1]
    y = np.abs(ref.norm_rope(x, w, None, None, (), eps, norm))
    P = sum(sections)
    both = y.copy()
    for p in range(P):
        i, j = (2 * p, 2 * p + 1) if inter else (p, p + P)
        both[..., i] = both[..., j] = y[..., i] + y[..., j]
    e = ((D + 16) * F32 + 2.0 ** -19) * both
    return e * (1 + U[dt]) + U[dt] * np.abs(want) + TINY[dt]


def run_rope(T, hq, hk, D, dt, sections=None, inter=False, norm=True, weights=True, layout="packed", inplace=False,
             t0=0, seed=0, offset=0):
    g = gen(seed)
    if sections is None:
        p = D // 2 // 3
        sections = (D // 2 - 2 * p, p, p)
    H = hq + 2 * hk
    buf = rnd(g, (T * H * D + offset,), dt, 2.0).to(DEV)[offset:]
    if layout == "packed":
        full = buf.view(T, H, D)
    else:
        full = buf.view(H, T, D).transpose(0, 1)
    q, k = full[:, :hq], full[:, hq:hq + hk]
    wq, wk = ((1 + rnd(g, (D,), dt, 0.2)).to(DEV) for _ in range(2)) if weights and norm else (None, None)
    axes = len(sections)
    pos = (torch.randint(0, 300, (T, max(axes, 1)), generator=g, dtype=torch.int64) + t0).to(torch.int32).to(DEV)
    pos = pos[:, :axes].contiguous()
    freq = tk.rope_frequencies(sections, device=DEV) if axes else None
    nf = f64(freq) if axes else []
    qn, kn = f64(q), f64(k)
    if inplace:
        qo, ko = tk.qk_norm_rope(q, k, wq, wk, pos, freq, sections, norm=norm, interleaved=inter, q_out=q, k_out=k)
    else:
        before = full.clone()
        qo, ko = tk.qk_norm_rope(q, k, wq, wk, pos, freq, sections, norm=norm, interleaved=inter)
        assert torch.equal(full, before)
    torch.cuda.synchronize()
    for got, x, w in ((qo, qn, wq), (ko, kn, wk)):
        w = None if w is None else f64(w)
        want = ref.norm_rope(x, w, f64(pos), nf, sections, 1e-6, norm, inter)
        check(got, want, rope_bound(x, w, f64(pos), nf, sections, 1e-6, norm, inter, dt, want), (T, hq, hk, D, dt))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,hq,hk,D", [(1, 8, 8, 64), (1, 1, 1, 2), (5, 3, 1, 80), (16, 16, 4, 128), (33, 4, 2, 96),
                                       (100, 8, 8, 64), (7, 2, 2, 30), (9, 5, 1, 256), (64, 1, 1, 16), (3, 40, 8, 72),
                                       (1000, 2, 1, 32)])
def test_rope_sizes(T, hq, hk, D, inter, dt):
    say("rope", T, hq, hk, D, inter, dt)
    for layout in ("packed", "heads"):
        run_rope(T, hq, hk, D, dt, inter=inter, layout=layout)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,sections", [(64, (32,)), (64, (8, 24)), (64, (4, 2, 2)), (64, ()), (77, (20, 10, 8)),
                                        (63, (5, 5, 5)), (128, (0, 64, 0)), (48, (0, 8, 16)), (1, ()), (64, (16, 8, 4)),
                                        (80, (24, 8, 0))])
def test_rope_sections(D, sections, inter):
    say("rope sections", D, sections, inter)
    for norm, weights in ((True, True), (True, False), (False, False)):
        run_rope(19, 3, 2, D, "fp16", sections, inter, norm, weights)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,D,offset", [(40, 64, 0), (17, 96, 1), (3, 50, 2), (1, 128, 4)])
def test_rope_in_place_and_unaligned(T, D, offset, inter):
    run_rope(T, 4, 2, D, "bf16", inter=inter, inplace=True, offset=offset)
    run_rope(T, 4, 2, D, "fp16", inter=inter, offset=offset, layout="heads")


def test_rope_late_positions():
    run_rope(50, 2, 2, 64, "fp16", t0=2 ** 31 - 1000)
    run_rope(50, 2, 2, 64, "fp16", t0=-(2 ** 31) + 5)


def test_rope_empty_heads_and_tokens():
    g = gen(11)
    x = rnd(g, (6, 2, 32), "fp16").to(DEV)
    pos, freq = torch.zeros((6, 1), dtype=torch.int32, device=DEV), tk.rope_frequencies((16,), device=DEV)
    a, b = tk.qk_norm_rope(x, x[:, :0], None, None, pos, freq, (16,))
    c, d = tk.qk_norm_rope(x[:, :0], x, None, None, pos, freq, (16,))
    assert b.numel() == 0 and c.numel() == 0 and torch.equal(a, d)
    e, _ = tk.qk_norm_rope(x[:0], x[:0], None, None, pos[:0], freq, (16,))
    assert e.shape == (0, 2, 32)


def test_rope_rows_of_zeros_infinities_and_nan():
    x = rnd(gen(12), (4, 2, 64), "fp16")
    x[0, 0] = 0.0
    x[1, 1, 5] = float("inf")
    x[2, 0, 7] = float("nan")
    pos = torch.arange(4, dtype=torch.int32).view(4, 1).to(DEV)
    y, _ = tk.qk_norm_rope(x.to(DEV), x.to(DEV), None, None, pos, tk.rope_frequencies((32,), device=DEV), (32,))
    y = y.cpu()
    assert bool((y[0, 0] == 0).all()) and torch.isnan(y[2, 0]).all() and torch.isnan(y[1, 1, 5])
    ok = [(0, 1), (1, 0), (2, 1), (3, 0), (3, 1)]
    want = ref.norm_rope(f64(x), None, f64(pos), f64(tk.rope_frequencies((32,), device=DEV)), (32,))
    for i, j in ok:
        assert np.abs(f64(y[i, j]) - want[i, j]).max() <= 2.0 ** -9


def test_rope_large_values_do_not_overflow_the_norm():
    x = torch.full((2, 1, 128), 6e4, dtype=torch.float16, device=DEV)
    pos = torch.zeros((2, 1), dtype=torch.int32, device=DEV)
    y, _ = tk.qk_norm_rope(x, x, None, None, pos, tk.rope_frequencies((64,), device=DEV), (64,))
    assert bool((y == 1.0).all())


# ---------------------------------------------------------------- attention with a decay
def decay_check(o, S, q, k, v, ld, S0, lengths, scale, dt, what):
    want, wS = ref.decay_attention(q, k, v, ld, S0, lengths, scale)
    mag, mS = ref.decay_attention(np.abs(q), np.abs(k), np.abs(v), ld, None if S0 is None else np.abs(S0), lengths,
                                  abs(scale))
    T = q.shape[1]
    # products of rounded scores and rounded states with 16-bit operands, fp32 sums over the sequence
    bound = U[dt] * np.abs(want) + (2 * U[dt] + (T + 256) * F32) * mag + TINY[dt]
    check(o, want, bound, what)
    rms = np.sqrt(((f64(o) - want) ** 2).mean() / max((want ** 2).mean(), 1e-300))
    assert rms <= U[dt], (what, rms)
    if S is not None:
        # the state is fp32: sums of the sequence's length, products to 2^-21
        assert S.dtype == torch.float32
        sb = ((T + 16) * F32 + 2.0 ** -21) * mS + 1e-37
        check(S, wS, sb, (what, "state"))


def run_decay(B, T, H, K, D, V, dt, decay="multi", ragged=None, state=True, layout="packed", want_state=True, offset=0,
              inplace=False, seed=0, scale=None, mag=1.0):
    g = gen(seed)

    def make(h, d):
        if layout == "heads":
            return rnd(g, (B * h * T * d + offset,), dt, mag).to(DEV)[offset:].view(B, h, T, d).transpose(1, 2)
        if layout == "time":  # tokens slowest
            return rnd(g, (B * h * T * d + offset,), dt, mag).to(DEV)[offset:].view(T, B, h, d).transpose(0, 1)
        pad = 5 if layout == "padded" else 0
        return rnd(g, (B * T * h * (d + pad) + offset,), dt, mag).to(DEV)[offset:].view(B, T, h, d + pad)[..., :d]

    q, k, v = make(H, D), make(K, D), make(K, V)
    i = torch.arange(H, dtype=torch.float64)
    lam = {"multi": 1 - 2.0 ** -(3 + 6 * i / max(H - 1, 1)), "strong": 0.02 + 0.6 * i / max(H - 1, 1),
           "none": torch.ones(H, dtype=torch.float64), "zero": torch.zeros(H, dtype=torch.float64),
           "mixed": torch.where(i % 2 == 0, 1.0, 1e-30)}[decay]
    ld = lam.log().float().to(DEV)
    S0 = (torch.randn((B, H, D, V), generator=g) * 3 * mag * mag).to(DEV) if state else None
    ln = None if ragged is None else torch.tensor(ragged, dtype=torch.int32, device=DEV)
    if ragged is not None:  # what lies past a sequence's end is never used
        for b, n in enumerate(ragged):
            n = min(max(n, 0), T)
            for x, bad in ((q, float("nan")), (k, float("inf")), (v, float("nan"))):
                x[b, n:] = bad
    sc = D ** -0.5 if scale is None else scale
    args = [f64(x) for x in (q, k, v)]
    if ragged is not None:
        args = [np.nan_to_num(a, nan=0.0, posinf=0.0) for a in args]
    S0n = None if S0 is None else f64(S0)
    out = torch.full((B, T, H, V), 9.0, dtype=DT[dt], device=DEV)
    got = tk.decay_attention(q, k, v, ld, S0, ln, sc, return_state=want_state, out=out,
                             state_out=S0 if inplace else None)
    torch.cuda.synchronize()
    o, S = got if want_state else (got, None)
    decay_check(o, S, *args, f64(ld), S0n, ragged, sc, dt, (B, T, H, K, D, V, dt, decay, ragged, layout))
    if ragged is not None:
        for b, n in enumerate(ragged):
            assert bool((o[b, max(n, 0):] == 0).all())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 3, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129, 200, 257, 515])
def test_decay_lengths(T, dt):
    say("decay", T, dt)
    run_decay(2, T, 4, 4, 64, 64, dt)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("D,V", [(1, 1), (16, 16), (32, 32), (64, 128), (128, 64), (128, 128), (40, 75), (75, 33),
                                 (96, 96), (127, 5), (8, 120), (33, 64)])
def test_decay_widths(D, V, dt):
    say("decay widths", D, V, dt)
    run_decay(1, 150, 2, 1, D, V, dt)
    run_decay(3, 1, 2, 2, D, V, dt)


@pytest.mark.parametrize("T", [1, 70, 300])
@pytest.mark.parametrize("H,K", [(1, 1), (6, 3), (8, 1), (5, 5)])
def test_decay_shared_heads(H, K, T):
    say("decay heads", H, K, T)
    run_decay(2, T, H, K, 32, 48, "fp16")


@pytest.mark.parametrize("T", [1, 40, 333])
@pytest.mark.parametrize("decay", ["strong", "none", "zero", "mixed"])
def test_decay_decays(decay, T):
    say("decay rates", decay, T)
    for dt in ("fp16", "bf16"):
        run_decay(2, T, 4, 2, 64, 64, dt, decay=decay)


@pytest.mark.parametrize("T,ragged", [(1, [1, 0, 1, 0]), (90, [90, 0, 1, 64]), (300, [300, 1, 129, 0]), (200, [0, 0, 0, 0]),
                                      (130, [1000, -5, 128, 127]), (700, [640, 641, 639, 13])])
def test_decay_ragged(T, ragged):
    say("decay ragged", T, ragged)
    for dt in ("fp16", "bf16"):
        run_decay(4, T, 2, 1, 64, 32, dt, ragged=ragged)
    run_decay(4, T, 2, 2, 128, 128, "fp16", ragged=ragged, state=False)


@pytest.mark.parametrize("T", [1, 77, 260])
@pytest.mark.parametrize("layout,offset", [("heads", 0), ("time", 0), ("padded", 0), ("packed", 1), ("heads", 3)])
def test_decay_layouts(layout, offset, T):
    say("decay layout", layout, offset, T)
    run_decay(3, T, 4, 2, 64, 64, "fp16", layout=layout, offset=offset)
    run_decay(2, T, 2, 2, 50, 30, "bf16", layout=layout, offset=offset)


@pytest.mark.parametrize("T", [0, 1, 100, 600])
def test_decay_state_options(T):
    run_decay(2, T, 2, 2, 64, 64, "fp16", inplace=True) if T else None
    run_decay(2, T, 2, 2, 64, 64, "bf16", state=False) if T else None
    run_decay(2, T, 2, 2, 64, 64, "fp16", state=False, want_state=False) if T else None
    run_decay(2, T, 2, 2, 64, 64, "fp16", want_state=False) if T else None
    if T == 0:  # no token: the state goes through unchanged, or is zero
        S0 = torch.randn((2, 3, 16, 8), device=DEV)
        z = torch.empty((2, 0, 3, 16), dtype=torch.float16, device=DEV)
        ld = torch.full((3,), -0.5, device=DEV)
        o, S = tk.decay_attention(z, z, z[..., :8], ld, S0, return_state=True)
        assert o.shape == (2, 0, 3, 8) and torch.equal(S, S0)
        o, S = tk.decay_attention(z, z, z[..., :8], ld, None, return_state=True)
        assert bool((S == 0).all())


@pytest.mark.parametrize("B,T,H,D", [(1, 1, 2, 64), (1, 5, 1, 32), (2, 64, 2, 64), (1, 2000, 1, 64), (1, 900, 3, 128)])
def test_decay_state_in_place_is_the_state_apart(B, T, H, D):
    # also where a sequence is cut into segments, which begin and end at different times
    g = gen(25)
    q, k, v = (rnd(g, (B, T, H, D), "fp16").to(DEV) for _ in range(3))
    ld = torch.full((H,), -0.01, device=DEV)
    S = torch.randn((B, H, D, D), generator=g).to(DEV)
    o, S1 = tk.decay_attention(q, k, v, ld, S, return_state=True)
    o2, S2 = tk.decay_attention(q, k, v, ld, S, return_state=True, state_out=S)
    assert S2.data_ptr() == S.data_ptr() and torch.equal(o, o2) and torch.equal(S1, S2)


@pytest.mark.parametrize("T", [1, 50, 400])
@pytest.mark.parametrize("mag", [2.0 ** -7, 40.0])
def test_decay_magnitudes(mag, T):
    # small and large values: scores and states leave the range where fp16 is accurate, or the range of fp16
    say("decay magnitude", mag, T)
    run_decay(1, T, 2, 2, 64, 64, "bf16", mag=mag)
    if mag < 1:
        run_decay(1, T, 2, 2, 64, 64, "fp16", mag=mag, scale=256.0)
    else:
        run_decay(1, T, 2, 2, 64, 64, "fp16", mag=mag, scale=2.0 ** -12)


@pytest.mark.parametrize("cuts", [(1, 1, 1), (64, 1, 64), (100, 33, 200, 7)])
def test_decay_in_parts_is_the_whole(cuts):
    # a sequence in parts, its state handed on, against the oracle over the whole
    g = gen(21)
    T = sum(cuts)
    q, k, v = (rnd(g, (2, T, 2, 64), "fp16").to(DEV) for _ in range(3))
    ld = torch.tensor([-0.01, -0.3], device=DEV)
    S, outs, at = None, [], 0
    for n in cuts:
        o, S = tk.decay_attention(q[:, at:at + n], k[:, at:at + n], v[:, at:at + n], ld, S, scale=0.125, return_state=True)
        outs.append(o)
        at += n
    torch.cuda.synchronize()
    decay_check(torch.cat(outs, 1), S, *(f64(x) for x in (q, k, v)), f64(ld), None, None, 0.125, "fp16", cuts)


def test_decay_long_sequence_few_heads():
    say("decay long")
    run_decay(1, 3001, 1, 1, 64, 64, "fp16")
    run_decay(1, 2600, 2, 1, 128, 128, "bf16", ragged=[2555])


def test_decay_positive_decays_count_as_none():
    g = gen(22)
    q, k, v = (rnd(g, (1, 70, 2, 32), "fp16").to(DEV) for _ in range(3))
    a = tk.decay_attention(q, k, v, torch.tensor([0.5, 0.0], device=DEV), return_state=True)
    b = tk.decay_attention(q, k, v, torch.tensor([0.0, 0.0], device=DEV), return_state=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_decay_nan_reaches_no_earlier_token_and_no_other_head():
    g = gen(23)
    q, k, v = (rnd(g, (2, 150, 2, 64), "fp16") for _ in range(3))
    ld = torch.tensor([-0.05, -0.2], device=DEV)
    clean = tk.decay_attention(*(x.to(DEV) for x in (q, k, v)), ld).cpu()
    v[0, 100, 1, 3] = float("nan")
    k[1, 149, 0, 2] = float("inf")
    got = tk.decay_attention(*(x.to(DEV) for x in (q, k, v)), ld).cpu()
    assert torch.equal(got[0, :, 0], clean[0, :, 0]) and torch.equal(got[1, :, 1], clean[1, :, 1])
    assert torch.isfinite(got[0, :64]).all() and torch.isfinite(got[1, :128]).all()
    assert torch.isnan(got[0, 100:, 1, 3]).all()
    # to the token: what came before in the same stretch, and the other columns, are as they were
    assert torch.equal(got[0, :100, 1], clean[0, :100, 1]) and torch.equal(got[1, :149, 0], clean[1, :149, 0])
    other = torch.arange(64) != 3
    assert torch.isfinite(got[0, :, 1][:, other]).all()


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T", [5, 90])
def test_decay_state_that_is_not_finite(T, dt):
    # an infinity in one column of the state stays in that column
    g = gen(24)
    q, k, v = (rnd(g, (1, T, 1, 64), dt).to(DEV) for _ in range(3))
    ld = torch.tensor([-0.05], device=DEV)
    S = torch.randn((1, 1, 64, 64), generator=g).to(DEV)
    clean = tk.decay_attention(q, k, v, ld, S).cpu()
    S[0, 0, 5, 40] = float("inf")
    got = tk.decay_attention(q, k, v, ld, S).cpu()
    other = torch.arange(64) != 40
    assert not torch.isfinite(got[0, :, 0, 40]).any()
    assert torch.equal(got[..., other], clean[..., other])


def test_decay_offsets_past_32_bits():
    ld_, T = (1 << 30) + 8, 4  # tokens 2 and 3 begin past 2^31 elements
    buf = torch.empty(3 * ld_ + 4096, dtype=torch.float16, device=DEV)
    q, k, v = (buf.as_strided((1, T, 2, 32), (0, ld_, 32, 1), 512 * i) for i in range(3))
    for i, x in enumerate((q, k, v)):
        x.copy_(rnd(gen(30 + i), (1, T, 2, 32), "fp16"))
    lam = torch.tensor([-0.1, -0.2], device=DEV)
    a = tk.decay_attention(q, k, v, lam, return_state=True)
    b = tk.decay_attention(q.contiguous(), k.contiguous(), v.contiguous(), lam, return_state=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_rope_more_tokens_than_a_launch_takes():
    T, last = (1 << 25) + 777, 2000  # eight tokens of 256 a workgroup, 17 GB
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    q = torch.ones((T, 1, 256), dtype=torch.float16, device=DEV)
    rows = rnd(gen(44), (last, 1, 256), "fp16").to(DEV)
    q[-last:] = rows
    pos = torch.arange(T, dtype=torch.int32, device=DEV).view(T, 1)
    freq = tk.rope_frequencies((128,), device=DEV)
    none = q[:, :0]
    tk.qk_norm_rope(q, none, None, None, pos, freq, (128,), q_out=q, k_out=none)
    want, _ = tk.qk_norm_rope(rows, rows[:, :0], None, None, pos[-last:].contiguous(), freq, (128,))
    assert torch.equal(q[-last:], want)


# ---------------------------------------------------------------- streams, graphs, refusals
def test_operators_replay_in_a_graph():
    g = gen(40)
    x = rnd(g, (200, 128), "fp16").to(DEV)
    w = rnd(g, (384, 128), "fp16", 0.1).to(DEV)
    pos = tk.grid_positions(1, 10, 20, device=DEV)
    freq = tk.rope_frequencies((8, 4, 4), device=DEV)
    ld = torch.tensor([-0.02, -0.1, -0.3, 0.0], device=DEV)
    state = torch.zeros((1, 4, 32, 32), device=DEV)

    def step():
        qkv = tk.linear(x, w).view(200, 12, 32)
        q, k = tk.qk_norm_rope(qkv[:, :4], qkv[:, 4:8], None, None, pos, freq, (8, 4, 4))
        return tk.decay_attention(q[None], k[None], qkv[None, :, 8:], ld, state, return_state=True, state_out=state)[0]

    eager = []
    for _ in range(4):
        eager.append(step().clone())
    final = state.clone()
    state.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    state.zero_()
    with torch.cuda.graph(graph):
        out = step()
    state.zero_()
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]), i
        torch.randn(1000, device=DEV).sum().item()  # other work between the replays
    assert torch.equal(state, final)


def test_refusals_of_tensors():
    x = torch.zeros((4, 64), dtype=torch.float16, device=DEV)
    w = torch.zeros((32, 64), dtype=torch.float16, device=DEV)
    for bad in (lambda: tk.linear(x.float(), w.float()), lambda: tk.linear(x, w.bfloat16()), lambda: tk.linear(x.cpu(), w),
                lambda: tk.linear(x, w[:, :63]), lambda: tk.linear(x.t(), w), lambda: tk.linear(x, w, act="tanh"),
                lambda: tk.linear(x, w[:31], gated=True), lambda: tk.linear(x, w, bias=w[0]),
                lambda: tk.linear(x, w, residual=x), lambda: tk.linear(x, w, out=x),
                lambda: tk.linear(torch.zeros((4, 6, 64), dtype=torch.float16, device=DEV)[:, :3], w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(nc.NcodecError) as e:
        tk.linear(x[:1].expand(4, 64), w)  # rows that are one row
    assert e.value.status == nc.NCODEC_ESHAPE
    q = torch.zeros((4, 2, 64), dtype=torch.float16, device=DEV)
    pos, fr = torch.zeros((4, 2), dtype=torch.int32, device=DEV), tk.rope_frequencies((8, 8), device=DEV)
    for bad in (lambda: tk.qk_norm_rope(q, q[:3]), lambda: tk.qk_norm_rope(q, q, None, None, pos, fr, (8,)),
                lambda: tk.qk_norm_rope(q, q, None, None, pos.long(), fr, (8, 8)),
                lambda: tk.qk_norm_rope(q, q, None, None, pos, fr[:-1], (8, 8)),
                lambda: tk.qk_norm_rope(q, q, None, None, None, fr, (8, 8)),
                lambda: tk.qk_norm_rope(q, q, q[0, 0], None, norm=False)):
        with pytest.raises(ValueError):
            bad()
    a = torch.zeros((1, 4, 2, 32), dtype=torch.float16, device=DEV)
    ld = torch.zeros(2, device=DEV)
    S = torch.zeros((1, 2, 32, 32), device=DEV)
    for bad in (lambda: tk.decay_attention(a, a, a, ld.half()), lambda: tk.decay_attention(a, a[:, :3], a, ld),
                lambda: tk.decay_attention(a, a, a, ld, S.transpose(2, 3)), lambda: tk.decay_attention(a, a, a, ld, S.half()),
                lambda: tk.decay_attention(a, a, a, ld, lengths=torch.zeros(2, dtype=torch.int32, device=DEV)),
                lambda: tk.decay_attention(a[0], a[0], a[0], ld)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(nc.NcodecError) as e:
        tk.decay_attention(torch.cat([a, a, a], 2)[:, :, :4].contiguous(), torch.cat([a, a], 2)[:, :, :3].contiguous(),
                           torch.cat([a, a], 2)[:, :, :3].contiguous(), torch.zeros(4, device=DEV))
    assert e.value.status == nc.NCODEC_ESHAPE  # 4 heads over 3 key heads
