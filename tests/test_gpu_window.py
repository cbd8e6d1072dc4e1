"""Softmax attention with a window and sinks on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

from attention_util import DEV, U, check, check_rounding, f64, gen, output_bound, rnd, say, sequences
from oracle import tokens as ref
from paper_2502_20762_amd import ncodec as nc
from paper_2502_20762_amd import tokens as tk

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def run(B, T, H, K, D, V, dt, window=None, sinks=0, lengths=None, layout="packed", offset=0, pad=0, seed=0, scale=None,
        mag=1.0):
    g = gen(seed)
    q, k, v = (sequences(g, B, T, h, d, dt, layout, offset, pad, mag if x else 1.0) for x, (h, d) in
               enumerate(((H, D), (K, D), (K, V))))
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    buf = torch.full((B, T, H, V + 3), 7.0, dtype=q.dtype, device=DEV)
    out = buf[..., 1:V + 1]
    sc = D ** -0.5 if scale is None else scale
    tk.window_attention(q, k, v, window, sinks, ln, scale, out=out)
    torch.cuda.synchronize()
    assert bool((buf[..., 0] == 7.0).all()) and bool((buf[..., V + 1:] == 7.0).all())
    qn, kn, vn = f64(q), f64(k), f64(v)
    want = ref.window_attention(qn, kn, vn, window, sinks, lengths, sc)
    size = ref.window_attention(qn, kn, np.abs(vn), window, sinks, lengths, sc)
    what = (B, T, H, K, D, V, dt, window, sinks)
    n = T if window is None else min(T, window + sinks)
    check(out, want, output_bound(want, size, np.abs(vn).max(), qn, kn, sc, D, n, dt), what)
    if want.size >= 4096:
        check_rounding(out, want, dt, what)
    return out


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 7, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 190, 257])
def test_lengths(T, dt):
    say("window", T, dt)
    run(2, T, 2, 1, 64, 64, dt)
    run(1, T, 2, 2, 64, 64, dt, window=max(1, T // 3), sinks=2)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("D,V", [(64, 64), (128, 128), (16, 16), (32, 96), (96, 32), (1, 1), (75, 33), (33, 75), (40, 128),
                                 (128, 7), (2, 100), (127, 127), (64, 128), (128, 64)])
@pytest.mark.parametrize("layout", ["packed", "heads"])
def test_widths(D, V, layout, dt):
    say("window", D, V, layout, dt)
    run(2, 90, 4, 2, D, V, dt, window=40, sinks=3, layout=layout)
    run(1, 150, 2, 1, D, V, dt, layout=layout)


@pytest.mark.parametrize("window", [None, 1, 2, 17, 32, 63, 64, 65, 130, 299, 300, 5000])
@pytest.mark.parametrize("sinks", [0, 1, 5, 31, 32, 64, 100, 1000])
def test_windows_and_sinks(window, sinks):
    say("window", window, sinks)
    run(1, 300, 2, 2, 32, 32, "fp16", window, sinks)


@pytest.mark.parametrize("window", [None, 1, 17, 40, 64, 130])
@pytest.mark.parametrize("sinks", [0, 5, 64, 100, 1000])
def test_windows_and_sinks_of_shared_heads(window, sinks):
    # waves on heads of a group: 32 queries a workgroup, which begin inside a tile of keys
    say("window shared", window, sinks)
    run(1, 300, 4, 1, 32, 32, "fp16", window, sinks)
    run(1, 300, 2, 1, 128, 32, "bf16", window, sinks)
    run(3, 140, 128, 2, 16, 128, "fp16", window, sinks)  # waves that do not share queries


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("window,sinks", [(None, 0), (50, 4), (200, 100)])
def test_ragged(window, sinks, dt):
    say("window ragged", window, sinks, dt)
    lengths = [260, 0, 1, 33, 64, 199, -5, 9000]
    o = run(8, 260, 4, 2, 64, 96, dt, window, sinks, lengths)
    for b, n in enumerate(lengths):
        assert bool((o[b, max(n, 0):] == 0).all())


@pytest.mark.parametrize("offset,pad", [(1, 0), (0, 1), (3, 5), (8, 8), (4, 4), (0, 8)])
@pytest.mark.parametrize("D", [64, 128])
def test_strides_and_alignment(D, offset, pad):
    run(2, 140, 2, 1, D, D, "fp16", 70, 5, None, "packed", offset, pad)
    run(2, 140, 2, 1, D, D, "bf16", None, 0, None, "heads", offset, pad)


@pytest.mark.parametrize("H,K", [(1, 1), (3, 1), (8, 2), (16, 1), (5, 5), (40, 8)])
def test_heads(H, K):
    run(2, 70, H, K, 64, 32, "fp16", 33, 2)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T,H,K,D,V,window,sinks", [(700, 2, 1, 128, 128, None, 0), (1000, 2, 2, 64, 64, 300, 40),
                                                    (1500, 1, 1, 128, 64, 511, 129)])
def test_long(T, H, K, D, V, window, sinks, dt):
    say("window long", T, H, K, D, V, window, sinks, dt)
    run(1, T, H, K, D, V, dt, window, sinks)


# padded widths, direct loads or not, and each with waves that share queries in halves or not: (batch, heads, kv_heads, head
# width, value width)
FORMS = {(D, V, halves): (B, H, K, D, V)
         for D in (64, 33, 128, 75) for V in (32, 64, 33, 96, 128, 100)
         for halves, B, H, K in ((True, 2, 4, 1), (False, 17 if D <= 64 and V <= 64 else 5, 32, 8))}


@pytest.mark.parametrize("form", FORMS)
def test_every_form(form):
    say("window form", form)
    B, H, K, D, V = FORMS[form]
    run(B, 130 if form[2] else 129, H, K, D, V, "fp16" if V % 64 else "bf16", 70, 3)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("what", [INF, NAN])
def test_what_is_not_finite_where_waves_do_not_share_queries(what, dt):
    g = gen(12)
    B, T, H, K = 5, 150, 32, 8
    x = [rnd(g, (B, T, h, 128), dt) for h in (H, K, K)]
    clean = tk.window_attention(*(t.to(DEV) for t in x), 60, 4).cpu()
    for i, at in ((1, 70), (2, 70), (2, 1), (2, 149)):
        y = [t.clone() for t in x]
        y[i][1, at, 5, 40] = what
        o = tk.window_attention(*(t.to(DEV) for t in y), 60, 4).cpu()
        hit = torch.zeros((B, T, H, 128), dtype=torch.bool)
        seen = torch.arange(T) >= at
        if at >= 4:
            seen &= torch.arange(T) < at + 60
        hit[1, seen, 20:24] = True
        if i == 2:
            hit &= torch.arange(128) == 40
        fine = torch.isfinite(o)
        if i == 2:
            assert torch.equal(fine, ~hit), (i, at)
        else:  # a score of -inf takes its token away, all others end the mean
            assert bool(fine[~hit].all()) and not bool(fine[hit].all())
        assert torch.equal(o[~hit], clean[~hit])


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_stretches_of_minus_infinity_and_nan_between_the_halves(dt):
    # tiles of 64 keys go to the two waves of a query in turn: whole tiles of one of them, or all of its own
    T = 500
    q = torch.ones((1, T, 1, 64), device=DEV).to(torch.float16 if dt == "fp16" else torch.bfloat16)
    v = rnd(gen(13), (1, T, 1, 64), dt).to(DEV)
    tile = torch.arange(T, device=DEV) // 64
    for gone in (tile % 2 == 0, tile % 2 == 1, tile < 3, tile == 7, tile < 8):
        k = torch.ones_like(q)
        k[0, gone] = -INF
        o = tk.window_attention(q, k, v, scale=0.01)
        with np.errstate(invalid="ignore"):
            want = ref.window_attention(f64(q), f64(k), f64(v), scale=0.01)
        assert np.array_equal(np.isfinite(f64(o)), np.isfinite(want))
        fine = np.isfinite(want)
        assert np.abs(f64(o) - want)[fine].max(initial=0) <= 2 * U[dt] * np.abs(f64(v)).max()
        k[0, gone] = NAN
        o = tk.window_attention(q, k, v, scale=0.01)
        first = int(gone.nonzero()[0])
        assert torch.isnan(o[0, first:]).all() and torch.isfinite(o[0, :first]).all()


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_peaked_and_flat_weights(dt):
    # scores of some hundreds: one token takes all; scale 0: all weigh the same
    run(1, 200, 2, 2, 64, 64, dt, None, 0, mag=6.0, scale=1.0)
    run(1, 200, 2, 2, 64, 64, dt, 64, 3, scale=0.0)
    run(1, 200, 2, 2, 64, 64, dt, 64, 3, scale=-0.3)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_maxima_that_rise_and_fall(dt):
    # the largest score of a token comes first, last, or grows from key to key by more than a fp16 weight's range
    T, D = 300, 32
    for rise in (0.5, -0.5):
        q, k = torch.zeros((1, T, 1, D)), torch.zeros((1, T, 1, D))
        q[..., 0] = 1.0
        k[..., 0] = rise * torch.arange(T).view(1, T, 1)
        v = torch.randn((1, T, 1, D), generator=gen(1))
        q, k, v = (x.to(torch.float16 if dt == "fp16" else torch.bfloat16) for x in (q, k, v))
        for window, sinks in ((None, 0), (100, 7)):
            o = tk.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), window, sinks, scale=1.0)
            args = (f64(q), f64(k))
            want = ref.window_attention(*args, f64(v), window, sinks)
            size = ref.window_attention(*args, np.abs(f64(v)), window, sinks)
            check(o, want, output_bound(want, size, np.abs(f64(v)).max(), *args, 1.0 / D, D, T, dt), (rise, window))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_values_at_the_end_of_the_range(dt):
    # a weighted mean of such values is one, however many they are
    top = {"fp16": 65504.0, "bf16": 3.3e38}[dt]
    T = 200
    q = rnd(gen(2), (1, T, 1, 64), dt).to(DEV)
    v = torch.full((1, T, 1, 64), top, device=DEV).to(q.dtype)
    v[..., 32:] *= -1
    o = tk.window_attention(q, q, v, scale=0.1)
    assert torch.isfinite(o).all()
    assert np.abs(f64(o) / f64(v) - 1).max() <= 2 * U[dt]


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("where", ["q", "k", "v"])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
@pytest.mark.parametrize("T,window,sinks", [(10, None, 0), (100, 30, 4), (300, 70, 9)])
def test_what_is_not_finite_reaches_who_sees_it(T, window, sinks, what, where, dt):
    # the outputs that are not finite are the formula's, and the others are what they are without it
    say("not finite", T, window, sinks, what, where, dt)
    g = gen(3)
    x = {n: rnd(g, (1, T, 2, 64), dt) for n in "qkv"}
    clean = tk.window_attention(*(x[n].to(DEV) for n in "qkv"), window, sinks, scale=0.125)
    for at in (0, T // 2, T - 1):
        y = {n: t.clone() for n, t in x.items()}
        y[where][0, at, 1, 40] = what
        o = tk.window_attention(*(y[n].to(DEV) for n in "qkv"), window, sinks, scale=0.125)
        with np.errstate(invalid="ignore"):
            want = ref.window_attention(*(f64(y[n]) for n in "qkv"), window, sinks, None, 0.125)
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(f64(o)), fine), at
        same = torch.from_numpy(fine) & torch.from_numpy(np.isclose(want, ref.window_attention(
            *(f64(x[n]) for n in "qkv"), window, sinks, None, 0.125), rtol=0, atol=0))
        assert torch.equal(o.cpu()[same], clean.cpu()[same])


def test_a_token_whose_scores_are_all_minus_infinity_is_no_number():
    q = torch.ones((1, 3, 1, 8), dtype=torch.float16, device=DEV)
    k = torch.full((1, 3, 1, 8), -INF, dtype=torch.float16, device=DEV)
    k[0, 2] = 1.0
    o = tk.window_attention(q, k, q)
    assert torch.isnan(o[0, :2]).all() and bool((o[0, 2] == 1).all())


@pytest.mark.parametrize("T", [40, 300])
def test_padding_is_not_used(T):
    g = gen(4)
    q, k, v = (rnd(g, (2, T, 2, 64), "fp16").to(DEV) for _ in range(3))
    ln = torch.tensor([T - 23, 5], dtype=torch.int32, device=DEV)
    a = tk.window_attention(q, k, v, 50, 3, ln)
    for x in (q, k, v):
        x[0, T - 23:], x[1, 5:] = NAN, INF
    b = tk.window_attention(q, k, v, 50, 3, ln)
    assert torch.equal(a, b) and torch.isfinite(a).all()


def test_a_sequence_does_not_depend_on_the_others_of_its_batch():
    # bit for bit, where the same number of workgroups takes both
    g = gen(14)
    q, k, v = (rnd(g, (4, 200, 2, 64), "bf16").to(DEV) for _ in range(3))
    whole = tk.window_attention(q, k, v, 90, 10)
    q[[0, 2, 3]], k[[0, 2, 3]], v[[0, 2, 3]] = 3 * q[[2, 3, 0]], -k[[3, 0, 2]], v[[3, 0, 2]]
    assert torch.equal(tk.window_attention(q, k, v, 90, 10)[1], whole[1])


def test_each_sequence_by_itself_and_prefixes_agree():
    g = gen(5)
    q, k, v = (rnd(g, (3, 333, 2, 64), "bf16").to(DEV) for _ in range(3))
    ln = torch.tensor([333, 100, 222], dtype=torch.int32, device=DEV)
    for window, sinks in ((None, 0), (90, 10)):
        whole = tk.window_attention(q, k, v, window, sinks, ln)
        for b, n in enumerate(ln.tolist()):
            one = tk.window_attention(*(x[b:b + 1, :n] for x in (q, k, v)), window, sinks)
            assert (one[0].float() - whole[b, :n].float()).abs().max() <= 4 * U["bf16"] * whole[b, :n].float().abs().max()


def test_empty_calls():
    x = torch.ones((2, 0, 2, 64), dtype=torch.float16, device=DEV)
    assert tk.window_attention(x, x, x).shape == (2, 0, 2, 64)
    x = torch.ones((0, 5, 2, 64), dtype=torch.float16, device=DEV)
    assert tk.window_attention(x, x, x).shape == (0, 5, 2, 64)


def test_rows_past_32_bit_offsets():
    ld = (1 << 26) + 64  # token 64 begins past 2^32 elements
    buf = torch.empty(70 * ld, dtype=torch.float16, device=DEV)
    x = rnd(gen(6), (1, 70, 2, 64), "fp16").to(DEV)
    y = buf.as_strided((1, 70, 2, 64), (0, ld, 64, 1))
    y.copy_(x)
    want = tk.window_attention(x, x, x, 20, 2)
    assert torch.equal(tk.window_attention(y, y, y, 20, 2), want)
    out = buf.as_strided((1, 70, 2, 64), (0, ld, 64, 1), 1024)
    assert torch.equal(tk.window_attention(x, x, x, 20, 2, out=out), want)


def test_shared_heads_by_a_stride_of_zero():
    g = gen(7)
    q, k = rnd(g, (1, 100, 4, 64), "fp16").to(DEV), rnd(g, (1, 100, 1, 64), "fp16").to(DEV)
    assert torch.equal(tk.window_attention(q, k.expand(1, 100, 4, 64), k.expand(1, 100, 4, 64), 40),
                       tk.window_attention(q, k, k, 40))


def test_more_blocks_than_a_launch_takes():
    # batch * heads of 2^22 short sequences
    B = 1 << 20
    x = torch.ones((B, 2, 4, 1), dtype=torch.float16, device=DEV)
    x[:, 1] = 2.0
    o = tk.window_attention(x, x, x, 1)
    assert torch.equal(o, x)


def test_stream_and_graph():
    g = gen(8)
    q, k, v = (rnd(g, (2, 400, 2, 64), "fp16").to(DEV) for _ in range(3))
    want = tk.window_attention(q, k, v, 100, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = tk.window_attention(q, k, v, 100, 4)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(b, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = tk.window_attention(q, k, v, 100, 4)
    for seed in (9, 10, 11):
        q.copy_(rnd(gen(seed), q.shape, "fp16"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, tk.window_attention(q, k, v, 100, 4))


def test_refusals():
    x = torch.ones((1, 4, 2, 64), dtype=torch.float16, device=DEV)
    for bad in (dict(window=0), dict(window=-3), dict(out=x.bfloat16()), dict(lengths=torch.ones(1, device=DEV)),
                dict(lengths=torch.ones(2, dtype=torch.int32, device=DEV)), dict(out=torch.empty_like(x[..., :5]))):
        with pytest.raises(ValueError):
            tk.window_attention(x, x, x, **bad)
    for bad in (lambda: tk.window_attention(x, x[:, :3], x), lambda: tk.window_attention(x, x, x[..., :0].float()),
                lambda: tk.window_attention(x.float(), x.float(), x.float()), lambda: tk.window_attention(x.cpu(), x, x),
                lambda: tk.window_attention(x, x[..., ::2], x), lambda: tk.window_attention(x[0], x[0], x[0])):
        with pytest.raises(ValueError):
            bad()
    wide = torch.ones((1, 4, 2, 129), dtype=torch.float16, device=DEV)
    for bad in (lambda: tk.window_attention(wide, wide, wide), lambda: tk.window_attention(x, x, x, sinks=-1),
                lambda: tk.window_attention(x, x, x, out=x), lambda: tk.window_attention(x, x, x, scale=INF),
                lambda: tk.window_attention(torch.cat([x, x[:, :, :1]], 2), x, x), lambda: tk.window_attention(x, x, x, window=1 << 31)):
        with pytest.raises(nc.NcodecError):
            bad()
    x.requires_grad_()
    y = x.detach()
    for args in ((x, y, y), (y, x, y), (y, y, x)):
        with pytest.raises(ValueError, match="no backward pass"):
            tk.window_attention(*args)
        with torch.no_grad():
            tk.window_attention(*args)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_window_values_that_are_no_numbers_count_however_small_their_weight(dt):
    # tiles of 64 keys go to two waves in turn; the low ones weigh exp(-512) of the others
    T, tile = 500, torch.arange(500, device=DEV) // 64
    q = torch.full((1, T, 1, 64), 8.0, device=DEV).to(torch.float16 if dt == "fp16" else torch.bfloat16)
    clean_v = torch.randn((1, T, 1, 64), device=DEV).to(q.dtype)
    for low in (tile % 2 == 0, tile % 2 == 1, tile < 3):
        k = torch.zeros_like(q)
        k[0, low] = -8.0
        at = int(low.nonzero()[5])
        v = clean_v.clone()
        v[0, at, 0, 3] = NAN
        o, clean = (tk.window_attention(q, k, x) for x in (v, clean_v))
        assert torch.isnan(o[0, at:, 0, 3]).all() and torch.isfinite(clean).all()
        o[0, at:, 0, 3] = clean[0, at:, 0, 3]
        assert torch.equal(o, clean)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", [1.1e3, 1e5, 3e5, 1.7e6, 1.3e7, -1.9e8, 3.3e12, 1e25])
def test_large_scores(scale, dt):
    # in fp32 they are further apart than powers of two: weights err, but no more than by their scores' rounding,
    # which is nothing where one token is ahead by more than that
    say("window large scores", scale, dt)
    g = gen(14)
    for B, T, H, K, D in ((1, 300, 2, 1, 64), (1, 150, 4, 4, 128), (3, 140, 128, 2, 16)):
        q, k, v = (rnd(g, (B, T, h, D), dt).to(DEV) for h in (H, K, K))
        for window, sinks in ((None, 0), (70, 3)):
            o = f64(tk.window_attention(q, k, v, window, sinks, scale=scale))
            want = ref.window_attention(f64(q), f64(k), f64(v), window, sinks, scale=scale)
            assert np.isfinite(o).all(), (T, window)
            top = np.abs(f64(v)).max()
            assert np.abs(o).max() <= top * (1 + 2 * U[dt])
            sure = ahead(f64(q), f64(k), scale, window, sinks)
            assert sure.mean() > 0.5
            assert np.abs(o - want)[sure].max() <= U[dt] * top * (1 + 2 * U[dt]) + 2.0 ** -15 * top, (T, window)


def ahead(q, k, scale, window, sinks):
    """(B, T, H): is one token ahead of all others by twice what fp32 scores err by, and 32 more?"""
    B, T, H, D = q.shape
    kk = np.repeat(k, H // k.shape[2], 2)
    s = scale * np.einsum("bihd,bjhd->bhij", q, kk)
    mag = abs(scale) * np.einsum("bihd,bjhd->bhij", np.abs(q), np.abs(kk)).max()
    i, j = np.arange(T)[:, None], np.arange(T)[None]
    s[..., ~((j <= i) & ((i - j < (window or T)) | (j < sinks)))] = -np.inf
    s.sort()
    second = np.where(np.isfinite(s[..., -2]), s[..., -2], s[..., -1] - 1e300)
    return (s[..., -1] - second > 2 * (D + 6) * 2.0 ** -24 * mag + 32).transpose(0, 2, 1)


@pytest.mark.parametrize("D,V", [(64, 64), (40, 96), (128, 128)])
@pytest.mark.parametrize("H,K", [(32, 8), (9, 3), (15, 15)])
def test_ragged_batches_of_many_blocks(H, K, D, V):
    # sequences take turns over the places of a launch, whatever number of them there is
    say("window many ragged", H, K, D, V)
    B = 10
    run(B, 150, H, K, D, V, "bf16", 70, 3, lengths=[(150, 0, 1)[b] if b < 3 else 37 * b % 151 for b in range(B)])
    run(1, 150, H, K, D, V, "fp16", None, 0, lengths=[131])
