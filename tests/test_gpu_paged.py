"""The paged cache on the GPU against the float64 oracle: attention of one new token, writes, eviction, and the run of them."""
import numpy as np
import pytest
import torch

from attention_util import (DEV, F32, U, Cache, check, check_rounding, f64, gen, output_bound, paged_reference, rnd, say,
                            sequences, weight_error)
from oracle import tokens as ref
from paper_2502_20762_amd import ncodec as nc
from paper_2502_20762_amd import tokens as tk

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------- attention of one token
def run(B, cap, H, K, D, V, dt, page=16, lengths=None, window=None, sinks=0, mass=False, layout="tokens", offset=0, seed=0,
        scale=None, fill=1.0, table=None):
    g = gen(seed)
    c = Cache(g, B, cap, page, K, D, V, dt, layout, extra_columns=seed % 3, fill=fill)
    q = rnd(g, (B * H * D + offset,), dt).to(DEV)[offset:].view(B, H, D)
    ln = i32([cap] * B if lengths is None else lengths)
    w = (torch.rand((B, K, c.columns), generator=g) * 3).to(DEV) if mass else None
    before = None if w is None else w.clone()
    buf = torch.full((B, H, V + 2), 7.0, dtype=q.dtype, device=DEV)
    sc = D ** -0.5 if scale is None else scale
    t = c.table if table is None else table(c.table)
    want, mag, wm = paged_reference(q, c, ln, window, sinks, sc, w, t)
    k0, v0 = c.k.clone(), c.v.clone()
    o = tk.paged_attention(q, c.k, c.v, t, ln, window, sinks, scale, w, out=buf[..., 1:V + 1])
    torch.cuda.synchronize()
    what = (B, cap, H, K, D, V, dt, page, window, sinks, layout)
    assert bool((buf[..., 0] == 7.0).all()) and bool((buf[..., V + 1:] == 7.0).all()), what
    assert torch.equal(k0, c.k) and torch.equal(v0, c.v)
    n = max([1] + ln.tolist())
    check(o, want, output_bound(want, mag, np.abs(f64(c.v)).max(), f64(q), f64(c.k), sc, D, n, dt), what)
    if want.size >= 2048:
        check_rounding(o, want, dt, what)
    if mass:
        e = 2 * weight_error(f64(q), f64(c.k), sc, D, "fp16") + (n + 64) * F32
        added = np.maximum(wm - f64(before), 0)
        check(w, wm, e * added + 2 * F32 * np.abs(wm), (what, "mass"))
        assert torch.equal(w[torch.from_numpy(added == 0).to(DEV)], before[torch.from_numpy(added == 0).to(DEV)])


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 1000, 5000])
def test_paged_lengths(n, dt):
    say("paged", n, dt)
    run(2, n, 2, 1, 64, 64, dt, mass=n % 2 == 0)
    run(3, n, 4, 4, 128, 128, dt, page=64, lengths=[n, n // 2, 1], window=max(1, n // 3), sinks=2, mass=True)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("D,V", [(64, 64), (128, 128), (16, 16), (32, 96), (96, 32), (1, 1), (75, 33), (33, 75), (40, 128),
                                 (128, 7), (2, 100), (127, 127), (64, 128), (128, 64)])
@pytest.mark.parametrize("layout", ["tokens", "heads", "beside"])
def test_paged_widths(D, V, layout, dt):
    say("paged", D, V, layout, dt)
    run(3, 200, 4, 2, D, V, dt, layout=layout, lengths=[200, 77, 0], mass=True)
    run(2, 700, 2, 1, D, V, dt, page=32, layout=layout, window=300, sinks=5, seed=1)


@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64, 128, 256, 1024, 4096])
def test_paged_page_sizes(page):
    run(3, 1500, 4, 2, 64, 64, "fp16", page=page, lengths=[1500, 1, 700], mass=True)
    run(2, 300, 2, 2, 32, 64, "bf16", page=page, window=120, sinks=9)


@pytest.mark.parametrize("window", [None, 1, 2, 17, 64, 130, 299, 300, 5000])
@pytest.mark.parametrize("sinks", [0, 1, 5, 32, 100, 1000])
def test_paged_windows_and_sinks(window, sinks):
    run(2, 300, 2, 1, 32, 32, "fp16", window=window, sinks=sinks, mass=True, lengths=[300, 150])


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("H,K", [(1, 1), (3, 1), (8, 2), (16, 1), (17, 1), (5, 5), (40, 8), (70, 2), (128, 1)])
def test_paged_heads(H, K, dt):
    say("paged heads", H, K, dt)
    run(2, 333, H, K, 64, 96, dt, lengths=[333, 50], mass=True)


@pytest.mark.parametrize("offset", [1, 4, 8])
@pytest.mark.parametrize("layout", ["tokens", "beside"])
def test_paged_alignment(offset, layout):
    run(2, 100, 4, 2, 64, 64 + offset, "fp16", offset=offset, layout=layout, mass=True)
    run(2, 100, 4, 2, 72 + offset, 64, "bf16", offset=offset, layout=layout)


def test_paged_ragged_lengths_out_of_range():
    run(6, 100, 2, 1, 64, 64, "fp16", lengths=[100, 0, -3, 1, 1000, 99], mass=True)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_paged_few_rows_over_a_long_cache(dt):
    say("paged long", dt)
    run(1, 40000, 4, 2, 64, 64, dt, page=128, mass=True)
    run(1, 30011, 2, 1, 128, 128, dt, page=64, window=20000, sinks=100)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_paged_many_rows(dt):
    run(300, 40, 8, 2, 64, 64, dt, lengths=[(7 * b) % 41 for b in range(300)], mass=True)


@pytest.mark.parametrize("mass", [False, True])
def test_paged_numbers_that_are_no_page_hold_nothing(mass):
    def spoil(t):
        t = t.clone()
        t[0, 1], t[0, 5], t[1, 0], t[2] = -1, 1 << 30, 99999, -(1 << 31)
        return t

    run(4, 300, 4, 2, 64, 64, "fp16", page=32, table=spoil, mass=mass)
    run(4, 300, 4, 2, 64, 64, "bf16", page=32, table=spoil, mass=mass, window=40, sinks=33)


def test_paged_pages_shared_by_sequences():
    run(4, 128, 4, 2, 64, 64, "fp16", page=32, table=lambda t: t[:1].expand(4, -1), mass=True, lengths=[128, 100, 64, 1])
    run(4, 128, 4, 2, 64, 64, "fp16", page=32, table=lambda t: t[:, :1].expand(-1, t.shape[1]).contiguous())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_paged_peaked_and_flat_weights(dt):
    run(2, 500, 2, 1, 64, 64, dt, fill=6.0, scale=1.0, mass=True)
    run(2, 500, 2, 1, 64, 64, dt, scale=0.0, mass=True)
    run(2, 500, 2, 1, 64, 64, dt, scale=-0.3)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_paged_values_at_the_end_of_the_range(dt):
    top = {"fp16": 65504.0, "bf16": 3.3e38}[dt]
    for n in (50, 20000):
        c = Cache(gen(2), 1, n, 16, 1, 64, 64, dt)
        c.v.fill_(top)
        c.v[..., 32:] *= -1
        q = rnd(gen(3), (1, 2, 64), dt).to(DEV)
        o = tk.paged_attention(q, c.k, c.v, c.table, i32([n]))
        assert torch.isfinite(o).all() and np.abs(f64(o) / f64(c.v[0, 0]) - 1).max() <= 2 * U[dt]


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("where", ["q", "k", "v"])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
@pytest.mark.parametrize("n,window,sinks", [(10, None, 0), (300, 70, 9), (3000, 1500, 9)])
def test_paged_what_is_not_finite_reaches_who_sees_it(n, window, sinks, what, where, dt):
    say("paged not finite", n, window, what, where, dt)
    g = gen(4)
    c = Cache(g, 2, n + 20, 16, 2, 64, 64, dt)
    q = rnd(g, (2, 4, 64), dt).to(DEV)
    ln = i32([n, n // 2])
    clean = tk.paged_attention(q, c.k, c.v, c.table, ln, window, sinks)
    for at in (0, n // 2, n - 1, n + 5):
        k, v, q2 = c.k.clone(), c.v.clone(), q.clone()
        page, row = int(c.table[0, at // 16]), at % 16
        if where == "q":
            q2[0, 3, 40] = what
        else:
            (k if where == "k" else v)[page, row, 1, 40] = what
        o = tk.paged_attention(q2, k, v, c.table, ln, window, sinks)
        with np.errstate(invalid="ignore"):
            want, _ = ref.paged_attention(f64(q2), f64(k), f64(v), f64(c.table).astype(np.int64), [n, n // 2], window, sinks,
                                          64 ** -0.5)
        assert np.array_equal(np.isfinite(f64(o)), np.isfinite(want)), at
        if where == "v" or what != what or where == "q":
            fine = torch.from_numpy(np.isfinite(want))
            assert torch.equal(o.cpu()[fine], clean.cpu()[fine]), at


def test_paged_rows_that_are_not_seen_are_not_used():
    # whatever the pages behind the last token hold, and those that the window has left
    g = gen(5)
    c = Cache(g, 2, 400, 32, 2, 64, 64, "fp16")
    q, ln = rnd(g, (2, 4, 64), "fp16").to(DEV), i32([333, 100])
    for window, sinks in ((None, 0), (90, 10)):
        a = tk.paged_attention(q, c.k, c.v, c.table, ln, window, sinks)
        for b, n in enumerate((333, 100)):
            j = np.setdiff1d(np.arange(c.columns), ref.seen(n - 1, window, sinks))
            p = c.table[b].cpu().numpy()[j // 32]
            for x in (c.k, c.v):
                x[torch.from_numpy(p).long().to(DEV), torch.from_numpy(j % 32).to(DEV)] = NAN
        assert torch.equal(a, tk.paged_attention(q, c.k, c.v, c.table, ln, window, sinks)) and torch.isfinite(a).all()


def test_paged_token_whose_scores_are_all_minus_infinity_is_no_number():
    c = Cache(gen(6), 1, 40, 16, 1, 64, 64, "fp16")
    c.k.fill_(-INF)
    mass = torch.zeros((1, 1, c.columns), device=DEV)
    o = tk.paged_attention(torch.ones((1, 1, 64), dtype=torch.float16, device=DEV), c.k, c.v, c.table, i32([40]), mass=mass)
    assert torch.isnan(o).all() and torch.isnan(mass[0, 0, :40]).all() and bool((mass[0, 0, 40:] == 0).all())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("n", [40, 3000])
def test_paged_stretches_of_nan_and_of_minus_infinity(n, dt):
    # a stretch as long as a wave's or a workgroup's share of the cache, the rest with scores that are numbers
    c = Cache(gen(6), 1, n, 16, 1, 64, 64, dt)
    q = torch.ones((1, 1, 64), dtype=c.k.dtype, device=DEV)
    t, page, row = c.table[0].long(), torch.arange(n, device=DEV) // 16, torch.arange(n, device=DEV) % 16
    for a, b in ((0, 32), (n // 2, n), (0, n - 1), (n - 1, n)):
        k = c.k.clone()
        k[t[page[a:b]], row[a:b]] = NAN
        assert torch.isnan(tk.paged_attention(q, k, c.v, c.table, i32([n]))).all(), (a, b)
        k[t[page[a:b]], row[a:b]] = -INF
        mass = torch.zeros((1, 1, c.columns), device=DEV)
        o = tk.paged_attention(q, k, c.v, c.table, i32([n]), mass=mass)
        want, mag, wm = paged_reference(q, Seen(c, k), i32([n]), None, 0, 0.125, mass * 0)
        check(o, want, output_bound(want, mag, np.abs(f64(c.v)).max(), f64(q), f64(c.k), 0.125, 64, n, dt), (a, b))
        assert bool((mass[0, 0, a:b] == 0).all()) and abs(float(mass.sum()) - 1) < 1e-4


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("n,low", [(40, 32), (3000, 1500), (3000, 2999), (20000, 9000)])
def test_paged_values_that_are_no_numbers_count_however_small_their_weight(n, low, dt):
    # `low` tokens, as many as a wave's or a workgroup's share, weigh exp(-512) of the others, or of the last one
    c = Cache(gen(6), 1, n, 16, 1, 64, 64, dt)
    q = torch.full((1, 1, 64), 8.0, dtype=c.k.dtype, device=DEV)
    t, j = c.table[0].long(), torch.arange(n, device=DEV)
    for key in (-8.0, -INF):
        c.k.zero_()
        c.k[t[j[:low] // 16], j[:low] % 16] = key
        v = c.v.clone()
        v[t[5 // 16], 5, 0, 3] = NAN
        o, clean = (tk.paged_attention(q, c.k, x, c.table, i32([n])) for x in (v, c.v))
        assert torch.isnan(o[0, 0, 3]) and torch.isfinite(clean).all()
        rest = torch.arange(64, device=DEV) != 3
        assert torch.equal(o[..., rest], clean[..., rest])


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", [1.1e3, 1e5, 3e5, 1.7e6, 1.3e7, -1.9e8, 3.3e12, 1e25])
def test_paged_large_scores(scale, dt):
    # in fp32 they are further apart than powers of two: weights err, but no more than by their scores' rounding,
    # which is nothing where one token is ahead by more than that
    say("paged large scores", scale, dt)
    g = gen(14)
    for B, n, H, K, D in ((8, 40, 4, 2, 64), (3, 3000, 32, 1, 128), (2, 20000, 2, 2, 64)):
        c = Cache(g, B, n, 16, K, D, 64, dt)
        q, ln, mass = rnd(g, (B, H, D), dt).to(DEV), i32([n] * B), torch.zeros((B, K, c.columns), device=DEV)
        o = f64(tk.paged_attention(q, c.k, c.v, c.table, ln, scale=scale))
        assert np.array_equal(o, f64(tk.paged_attention(q, c.k, c.v, c.table, ln, scale=scale, mass=mass)))
        want, _, wm = paged_reference(q, c, ln, None, 0, scale, mass * 0)
        top = np.abs(f64(c.v)).max()
        assert np.isfinite(o).all() and np.abs(o).max() <= top * (1 + 2 * U[dt])
        assert bool(torch.isfinite(mass).all()) and np.abs(f64(mass.sum(-1)) - H // K).max() < 1e-3 * (H // K)
        t = f64(c.table).astype(np.int64)[:, np.arange(n) // 16]
        k = f64(c.k)[t, np.arange(n) % 16]  # (B, n, K, D)
        kk = np.repeat(k, H // K, 2)
        s = scale * np.einsum("bhd,bjhd->bhj", f64(q), kk)
        mag = abs(scale) * np.einsum("bhd,bjhd->bhj", np.abs(f64(q)), np.abs(kk)).max()
        last = np.sort(s)[..., -2:]
        sure = last[..., 1] - last[..., 0] > 2 * (D + 6) * F32 * mag + 32
        assert np.abs(o - want)[sure].max(initial=0) <= U[dt] * top * (1 + 2 * U[dt]) + 2.0 ** -15 * top


class Seen:
    """A cache with other keys."""

    def __init__(self, c, k):
        self.k, self.v, self.table = k, c.v, c.table


def test_paged_offsets_past_32_bits():
    ld = (1 << 27) + 64  # page 40 begins past 2^32 elements
    buf = torch.empty(41 * ld + 4096, dtype=torch.float16, device=DEV)
    g = gen(7)
    c = Cache(g, 1, 41 * 16, 16, 1, 64, 64, "fp16", spare=0)
    k = buf.as_strided((41, 16, 1, 64), (ld, 64, 64, 1))
    v = buf.as_strided((41, 16, 1, 64), (ld, 64, 64, 1), 1 << 20)
    q, ln = rnd(g, (1, 2, 64), "fp16").to(DEV), i32([41 * 16])
    want = tk.paged_attention(q, c.k, c.v, c.table, ln)
    k.zero_()
    v.zero_()
    rows = [torch.stack([x[int(c.table[0, j // 16]), j % 16] for j in range(41 * 16)])[None] for x in (c.k, c.v)]
    tk.cache_append(rows[0], rows[1], k, v, c.table, i32([0]))
    assert torch.equal(k, c.k) and torch.equal(v, c.v)
    assert torch.equal(tk.paged_attention(q, k, v, c.table, ln), want)


def test_paged_without_pages_columns_or_sequences():
    x = torch.ones((2, 4, 64), dtype=torch.float16, device=DEV)
    c = Cache(gen(8), 2, 32, 16, 2, 64, 32, "fp16")
    none = torch.zeros((2, 0), dtype=torch.int32, device=DEV)
    for k, v, t in ((c.k[:0], c.v[:0], c.table), (c.k, c.v, none), (c.k[:0], c.v[:0], none)):
        m = torch.ones((2, 2, 16 * t.shape[1]), device=DEV)
        o = tk.paged_attention(x, k, v, t, i32([7, 0]), mass=m)
        assert bool((o == 0).all()) and o.shape == (2, 4, 32) and bool((m == 1).all())
        tk.cache_append(torch.ones((2, 3, 2, 64), dtype=torch.float16, device=DEV), torch.ones((2, 3, 2, 32), dtype=torch.float16, device=DEV),
                        k, v, t, i32([0, 1]), mass=m)
    assert tk.paged_attention(x[:0], c.k, c.v, c.table[:0], i32([])).shape == (0, 4, 32)


def test_paged_columns_behind_the_last_token_may_hold_anything():
    g = gen(9)
    for page in (1, 8, 16, 32):
        c = Cache(g, 2, 96, page, 2, 64, 64, "fp16")
        q, ln = rnd(g, (2, 4, 64), "fp16").to(DEV), i32([33, 1])
        a = tk.paged_attention(q, c.k, c.v, c.table, ln)
        for junk in (-1, 2 ** 31 - 1, 0, c.pages):
            t = c.table.clone()
            for b, n in enumerate((33, 1)):
                t[b, -(-n // page):] = junk
            assert torch.equal(a, tk.paged_attention(q, c.k, c.v, t, ln)), (page, junk)


# ---------------------------------------------------------------- writes
def run_append(B, T, K, D, V, dt, page=16, before=None, counts=None, mass=True, layout="tokens", rows="packed", offset=0,
               seed=0, spoil=None, columns=None):
    g = gen(seed)
    before = [5 * b for b in range(B)] if before is None else before
    c = Cache(g, B, columns or (max(before) + T), page, K, D, V, dt, layout, extra_columns=seed % 2)
    k, v = (sequences(g, B, T, K, d, dt, rows, offset) for d in (D, V))
    w = torch.rand((B, K, c.columns), generator=g).to(DEV) + 1 if mass else None
    t = c.table if spoil is None else spoil(c.table)
    n = None if counts is None else i32(counts)
    want = ref.cache_append(f64(k), f64(v), f64(c.k), f64(c.v), t.cpu().numpy(), before, counts, None if w is None else f64(w))
    tk.cache_append(k, v, c.k, c.v, t, i32(before), n, w)
    torch.cuda.synchronize()
    assert np.array_equal(f64(c.k), want[0]) and np.array_equal(f64(c.v), want[1])
    if mass:
        assert np.array_equal(f64(w), want[2])


@pytest.mark.parametrize("T", [1, 2, 7, 16, 33, 100, 1000])
@pytest.mark.parametrize("layout", ["tokens", "heads", "beside"])
def test_append_sizes(T, layout):
    say("append", T, layout)
    run_append(3, T, 2, 64, 64, "fp16", layout=layout)
    run_append(2, T, 4, 128, 128, "bf16", page=64, layout=layout, rows="heads", counts=[T, T // 2], mass=False)


@pytest.mark.parametrize("D,V", [(1, 1), (75, 33), (8, 16), (40, 128), (128, 7), (127, 127), (6, 20)])
@pytest.mark.parametrize("offset", [0, 1])
def test_append_widths(D, V, offset):
    for layout in ("tokens", "heads", "beside"):
        run_append(3, 21, 3, D, V, "fp16", layout=layout, offset=offset)


@pytest.mark.parametrize("page", [1, 2, 32, 256, 4096])
def test_append_page_sizes(page):
    run_append(3, 50, 2, 64, 32, "bf16", page=page, before=[0, 31, 300])


def test_append_what_falls_outside_goes_nowhere():
    run_append(6, 20, 2, 64, 64, "fp16", before=[0, -7, 90, 2 ** 31 - 5, -(2 ** 31), 95], columns=96,
               counts=[20, 20, 50, 20, 20, -3])

    def spoil(t):
        t = t.clone()
        t[0, 0], t[1, 1], t[2] = -1, 99999, 1 << 30
        return t

    run_append(4, 40, 2, 64, 64, "fp16", spoil=spoil)


def test_append_long():
    run_append(1, 20000, 2, 64, 64, "fp16", page=128)
    run_append(200, 3, 4, 32, 64, "bf16", counts=[b % 4 for b in range(200)])


# ---------------------------------------------------------------- eviction
def weights(g, shape, kind):
    w = torch.rand(shape, generator=g)
    if kind == "ties":
        w = (w * 4).floor()
    elif kind == "zeros":
        w = torch.zeros(shape)
    elif kind == "signs":
        w = torch.randn(shape, generator=g)
        w[w.abs() < 0.3] = 0.0
        w[torch.rand(shape, generator=g) < 0.1] = -0.0
    elif kind == "odd":
        w = torch.randn(shape, generator=g)
        for p, x in ((0.05, NAN), (0.05, INF), (0.05, -INF), (0.05, 1e-45), (0.05, -NAN)):
            w[torch.rand(shape, generator=g) < p] = x
    elif kind == "heavy":
        w = 1 / w - 1
    return w


def run_evict(B, cap, K, D, V, dt, keep, sinks=0, recent=0, page=16, lengths=None, kind="heavy", layout="tokens", seed=0,
              spoil=None, columns=None):
    g = gen(seed)
    c = Cache(g, 2 * B, max(cap, keep), page, K, D, V, dt, layout)
    table = c.table[:B, :-(-cap // page)]
    new = c.table[B:, :-(-(columns or keep) // page)]
    if spoil is not None:
        table, new = spoil(table.clone(), new.clone())
    ln = i32([cap] * B if lengths is None else lengths)
    w = weights(g, (B, K, table.shape[1] * page), kind).to(DEV)
    want = ref.cache_evict(f64(c.k), f64(c.v), table.cpu().numpy(), ln.tolist(), w.cpu().numpy(), keep, new.cpu().numpy(),
                           sinks, recent)
    w0 = w.clone()
    got = tk.cache_evict(c.k, c.v, table, ln, w, keep, new, sinks, recent)
    torch.cuda.synchronize()
    what = (B, cap, K, keep, sinks, recent, kind)
    assert np.array_equal(got[0].cpu().numpy(), want[2]), what
    assert np.array_equal(got[2].cpu().numpy(), want[4]), what
    assert np.array_equal(got[1].cpu().numpy(), want[3], equal_nan=True), what
    assert np.array_equal(f64(c.k), want[0]) and np.array_equal(f64(c.v), want[1]), what
    assert torch.equal(w0.view(torch.int32), w.view(torch.int32))


@pytest.mark.parametrize("kind", ["heavy", "ties", "zeros", "signs", "odd"])
@pytest.mark.parametrize("cap,keep,sinks,recent", [(1, 1, 0, 0), (5, 3, 1, 1), (64, 64, 0, 0), (65, 64, 64, 0), (65, 64, 0, 64),
                                                   (100, 40, 7, 13), (300, 200, 0, 0), (300, 1, 0, 0), (1000, 999, 3, 4),
                                                   (300, 20, 10, 10), (2100, 700, 16, 100)])
def test_evict_sizes(cap, keep, sinks, recent, kind):
    say("evict", cap, keep, sinks, recent, kind)
    run_evict(2, cap, 2, 64, 64, "fp16", keep, sinks, recent, kind=kind)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("D,V", [(1, 1), (75, 33), (8, 16), (40, 128), (128, 128), (127, 127)])
@pytest.mark.parametrize("layout", ["tokens", "heads", "beside"])
def test_evict_widths(D, V, layout, dt):
    # in one launch, and the rows in a launch of their own
    run_evict(2, 90, 3, D, V, dt, 33, 2, 5, layout=layout)
    run_evict(1, 5000, 2, D, V, dt, 1700, 20, 50, page=64, layout=layout, lengths=[4900])


def test_evict_ragged():
    for keep, sinks, recent in ((50, 4, 10), (99, 50, 49), (100, 0, 0)):
        run_evict(8, 100, 2, 64, 32, "fp16", keep, sinks, recent, lengths=[100, 0, 1, keep, keep + 1, -4, 1000, 52], kind="ties")


@pytest.mark.parametrize("page", [1, 2, 64, 1024])
def test_evict_page_sizes_and_room_to_spare(page):
    run_evict(2, 300, 2, 64, 64, "bf16", 120, 3, 9, page=page, columns=300)


def test_evict_numbers_that_are_no_page():
    def spoil(table, new):
        table[0, 1], table[1, 0], new[0, 0], new[1, 2] = -1, 99999, 1 << 30, -5
        return table, new

    run_evict(2, 200, 2, 64, 64, "fp16", 100, 3, 9, spoil=spoil)


@pytest.mark.parametrize("kind", ["heavy", "ties", "zeros", "signs", "odd"])
def test_evict_long(kind):
    # longer than a workgroup's share of 8192 positions, ends before, at and after it
    say("evict long", kind)
    run_evict(1, 20000, 2, 16, 16, "fp16", 7000, 64, 1000, page=128, kind=kind)
    lengths = [25000, 8191, 8192, 8193, 100, 16384, 0, 24577]
    run_evict(8, 25000, 1, 8, 8, "bf16", 9000, 0, 0, page=64, lengths=lengths, kind=kind)
    run_evict(2, 25000, 1, 8, 8, "fp16", 20000, 9000, 10000, page=64, lengths=[25000, 24000], kind=kind)
    run_evict(2, 17000, 1, 8, 8, "fp16", 9000, 4500, 4500, page=8, lengths=[17000, 9001], kind=kind)


def test_evict_of_nothing():
    c = Cache(gen(1), 2, 64, 16, 1, 8, 8, "fp16")
    none = torch.zeros((2, 0), dtype=torch.int32, device=DEV)
    k = c.k.clone()
    n, m, kept = tk.cache_evict(c.k, c.v, none, i32([5, 0]), torch.zeros((2, 1, 0), device=DEV), 3, c.table)
    assert n.tolist() == [0, 0] and bool((m == 0).all()) and bool((kept == -1).all()) and torch.equal(k, c.k)
    n, m, kept = tk.cache_evict(c.k, c.v, c.table[:0], i32([]), torch.zeros((0, 1, 64), device=DEV), 3, c.table[:0])
    assert n.shape == (0,) and m.shape == (0, 1, 64) and kept.shape == (0, 1, 3)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 5)])
def test_a_prompt_and_its_tokens_one_by_one_agree(window, sinks, dt):
    # an encoder has all tokens at once, a decoder each after the one before
    g = gen(9)
    B, T, H, K, D, V = 3, 120, 4, 2, 64, 32
    q, k, v = rnd(g, (B, T, H, D), dt).to(DEV), rnd(g, (B, T, K, D), dt).to(DEV), rnd(g, (B, T, K, V), dt).to(DEV)
    c = Cache(g, B, T, 16, K, D, V, dt)
    prompt = tk.window_attention(q, k, v, window, sinks)
    n = 70
    tk.cache_append(k[:, :n], v[:, :n], c.k, c.v, c.table, i32([0] * B))
    got = []
    for t in range(n, T):
        at = i32([t] * B)
        tk.cache_append(k[:, t:t + 1], v[:, t:t + 1], c.k, c.v, c.table, at)
        got.append(tk.paged_attention(q[:, t], c.k, c.v, c.table, at + 1, window, sinks))
    got = torch.stack(got, 1).float()
    # two roundings of the same values
    assert ((got - prompt[:, n:].float()).abs() <= 2.02 * U[dt] * prompt[:, n:].float().abs() + 2.0 ** -10 * U[dt]).all()


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_a_stream_with_a_budget(dt):
    """Tokens come one by one, their weights are summed, and whenever a stream is full it is cut back: step by step what
    the oracle does with the same cache."""
    g = gen(10)
    B, H, K, D, V, page, room, keep = 2, 4, 2, 32, 64, 16, 48, 24
    c = Cache(g, 2 * B, room, page, K, D, V, dt, spare=0)
    tables = [c.table[:B].contiguous(), c.table[B:].contiguous()]
    n = i32([0] * B)
    mass = torch.zeros((B, K, room), device=DEV)
    for t in range(110):
        q, k, v = rnd(g, (B, H, D), dt, 1.5).to(DEV), rnd(g, (B, 1, K, D), dt).to(DEV), rnd(g, (B, 1, K, V), dt).to(DEV)
        tk.cache_append(k, v, c.k, c.v, tables[0], n, mass=mass)
        n = n + 1
        want, mag, wm = paged_reference(q, c, n, None, 0, D ** -0.5, mass, tables[0])
        before = f64(mass)
        o = tk.paged_attention(q, c.k, c.v, tables[0], n, mass=mass)
        check(o, want, output_bound(want, mag, np.abs(f64(c.v)).max(), f64(q), f64(c.k), D ** -0.5, D, room, dt), t)
        e = 2 * weight_error(f64(q), f64(c.k), D ** -0.5, D, "fp16") + (room + 64) * F32
        check(mass, wm, e * np.maximum(wm - before, 0) + 2 * F32 * np.abs(wm), (t, "mass"))
        if int(n[0]) == room:
            want = ref.cache_evict(f64(c.k), f64(c.v), tables[0].cpu().numpy(), n.tolist(), mass.cpu().numpy(), keep,
                                   tables[1].cpu().numpy(), 2, 8)
            n, mass, kept = tk.cache_evict(c.k, c.v, tables[0], n, mass, keep, tables[1], 2, 8)
            tables.reverse()
            assert np.array_equal(f64(c.k), want[0]) and np.array_equal(f64(c.v), want[1])
            assert n.tolist() == want[2].tolist() and np.array_equal(mass.cpu().numpy(), want[3])
            assert np.array_equal(kept.cpu().numpy(), want[4])
            assert kept[:, :, :2].tolist() == [[[0, 1]] * K] * B and bool((kept[:, :, -8:] == torch.arange(40, 48, device=DEV)).all())


def test_streams_and_graph():
    # a step of a decoder, captured: write, attend, count; replayed beside the same steps made eagerly
    g = gen(11)
    B, H, K, D, T = 3, 4, 2, 64, 200
    a, b = (Cache(gen(12), B, T, 16, K, D, D, "fp16") for _ in range(2))
    q, k, v = (rnd(g, (B, 1, h, D), "fp16").to(DEV) for h in (H, K, K))
    n1, n2 = i32([100, 0, 37]), i32([100, 0, 37])
    m1, m2 = (torch.zeros((B, K, a.columns), device=DEV) for _ in range(2))

    def step(c, n, m):
        tk.cache_append(k, v, c.k, c.v, c.table, n, mass=m)
        n.add_(1)
        return tk.paged_attention(q[:, 0], c.k, c.v, c.table, n, window=90, sinks=4, mass=m)

    step(a, n1, m1)
    step(b, n2, m2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(a, n1, m1)
    for t in range(6):
        for x in (q, k, v):
            x.copy_(rnd(g, x.shape, "fp16"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(b, n2, m2)), t
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(m1, m2) and torch.equal(n1, n2)
    new = torch.arange(a.pages, a.pages + 3 * 4, dtype=torch.int32, device=DEV).view(3, 4)
    ks, vs = (torch.cat([x, torch.zeros_like(x[:12])]) for x in (a.k, a.v))
    want = [x.clone() for x in tk.cache_evict(ks, vs, a.table, n1, m1, 50, new, 2, 9)]
    wk = ks.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = tk.cache_evict(ks, vs, a.table, n1, m1, 50, new, 2, 9)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and torch.equal(ks, wk)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = tk.cache_evict(ks, vs, a.table, n1, m1, 50, new, 2, 9)
    for _ in range(3):
        m1.copy_(torch.rand(m1.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        copies = [x.clone() for x in (*got, ks, vs)]
        ks[a.pages:], vs[a.pages:] = 0, 0
        again = tk.cache_evict(ks, vs, a.table, n1, m1, 50, new, 2, 9)
        rows = [torch.equal(x, y) for x, y in zip(copies, (*again, ks, vs))]
        assert rows == [True] * 3 + rows[3:]
        for b_, count in enumerate(again[0].tolist()):
            j = torch.arange(count, device=DEV)
            p = new[b_, j // 16].long()
            assert torch.equal(copies[3][p, j % 16], ks[p, j % 16]) and torch.equal(copies[4][p, j % 16], vs[p, j % 16])


def test_refusals():
    c = Cache(gen(13), 2, 64, 16, 2, 64, 32, "fp16")
    q, ln = torch.ones((2, 4, 64), dtype=torch.float16, device=DEV), i32([3, 4])
    k, v = torch.ones((2, 1, 2, 64), dtype=torch.float16, device=DEV), torch.ones((2, 1, 2, 32), dtype=torch.float16, device=DEV)
    m = torch.zeros((2, 2, 64), device=DEV)
    new = c.table.clone()
    tk.paged_attention(q, c.k, c.v, c.table, ln, mass=m)
    for bad in (lambda: tk.paged_attention(q[0], c.k, c.v, c.table, ln), lambda: tk.paged_attention(q, c.k[0], c.v, c.table, ln),
                lambda: tk.paged_attention(q[..., :63], c.k, c.v, c.table, ln),
                lambda: tk.paged_attention(q, c.k, c.v, c.table.long(), ln),
                lambda: tk.paged_attention(q, c.k, c.v, c.table, ln.long()),
                lambda: tk.paged_attention(q, c.k, c.v, c.table, ln, mass=m[..., :63]),
                lambda: tk.paged_attention(q, c.k, c.v, c.table, ln, mass=m.double()),
                lambda: tk.paged_attention(q, c.k, c.v, c.table[0], ln), lambda: tk.paged_attention(q, c.k, c.v.float(), c.table, ln),
                lambda: tk.paged_attention(q, c.k, c.v, c.table, ln, window=0),
                lambda: tk.cache_append(k[0], v, c.k, c.v, c.table, ln), lambda: tk.cache_append(k, v[..., :3], c.k, c.v, c.table, ln),
                lambda: tk.cache_append(k.bfloat16(), v.bfloat16(), c.k, c.v, c.table, ln),
                lambda: tk.cache_append(k, v, c.k, c.v, c.table, ln, counts=ln[:1]),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, m, 65, new), lambda: tk.cache_evict(c.k, c.v, c.table, ln, m, 0, new),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, m, 5, new, out=(ln, m)),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln[:1], m, 5, new)):
        with pytest.raises(ValueError):
            bad()
    odd = torch.ones((4, 24, 2, 64), dtype=torch.float16, device=DEV)
    for bad in (lambda: tk.paged_attention(q[:, :3], c.k, c.v, c.table, ln), lambda: tk.paged_attention(q, c.k, c.v, c.table, ln, sinks=-1),
                lambda: tk.paged_attention(q, odd, odd, c.table, ln), lambda: tk.paged_attention(q, c.k, c.v, c.table, ln, scale=NAN),
                lambda: tk.paged_attention(q, q[:, None, :, :], q[:, None, :, :], c.table[:, :1], ln, out=q),
                lambda: tk.cache_append(c.k[:2, :1], v, c.k, c.v, c.table, ln),
                lambda: tk.cache_append(k, v, c.k[:1].expand(4, -1, -1, -1), c.v[:4], c.table, ln),
                lambda: tk.cache_append(k, k, c.k, c.k, c.table, ln),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, m, 5, new, sinks=3, recent=3),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, m, 5, new, sinks=-1),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, m, 5, new, out=(ln, torch.empty_like(m), torch.empty((2, 2, 5), dtype=torch.int32, device=DEV)))):
        with pytest.raises(nc.NcodecError):
            bad()
    x = q.clone().requires_grad_()
    with pytest.raises(ValueError, match="no backward pass"):
        tk.paged_attention(x, c.k, c.v, c.table, ln)
    for i in range(4):
        t = [k.clone(), v.clone(), c.k.clone(), c.v.clone()]
        t[i].requires_grad_()
        with pytest.raises(ValueError, match="no backward pass"):
            tk.cache_append(*t, c.table, ln)
        if i >= 2:
            with pytest.raises(ValueError, match="no backward pass"):
                tk.paged_attention(q, *t[2:], c.table, ln)
            with pytest.raises(ValueError, match="no backward pass"):
                tk.cache_evict(*t[2:], c.table, ln, m, 5, new)
