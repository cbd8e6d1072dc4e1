"""Values at both ends of bf16's range: a weighted mean of them is one of them, or lies between them.

Sums of weighted values are fp32 with the largest weight held below 1, at 2^-14 or above where one token has all the weight,
so that a product with a value of 2^-126 has its last bit at 2^-149: an addition of it errs by 2^-150, which is 2^-136 of an
output, and there are two for the two terms of the weight.  Halved steps of bf16 there are 2^-134."""
import numpy as np
import pytest
import torch

from attention_util import DEV, Cache, U, f64, gen, rnd, say
from paper_2502_20762_amd import tokens as tk
from test_gpu_paged import i32

pytestmark = pytest.mark.gpu

BF, HALF_STEP = torch.bfloat16, 2.0 ** -134


def small(g, shape, power):
    """bf16 numbers of both signs between 2^power and 2^(power + 1)."""
    x = torch.randint(128, 256, shape, generator=g).double() * torch.where(torch.rand(shape, generator=g) < 0.5, -1.0, 1.0)
    return (x * 2.0 ** (power - 7)).to(BF)


def peaked(T, D, at):
    """Queries and keys whose scores, scale 1, are 0 but for key `at`: 512, past the range of exp, for the tokens from it on;
    one token has all the weight."""
    q, k = torch.zeros((1, T, 1, D), dtype=BF), torch.zeros((1, T, 1, D), dtype=BF)
    q[..., 0] = 32.0
    k[0, at, 0, 0] = 16.0
    return q, k


@pytest.mark.parametrize("power", [-90, -101, -105, -109, -112, -117, -120, -125, -126])
@pytest.mark.parametrize("D,T", [(64, 40), (64, 300), (128, 300), (32, 2500)])
def test_window_one_token_has_all_the_weight(D, T, power):
    say("window small", D, T, power)
    v = small(gen(1), (1, T, 1, D), power)
    for at in (0, T // 3, T - 1):
        q, k = peaked(T, D, at)
        o = f64(tk.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=1.0))[0, at:, 0]
        want = f64(v)[0, at, 0]
        assert (np.abs(o - want) <= U["bf16"] * np.abs(want) + HALF_STEP + 2 * 2.0 ** -136).all(), at


@pytest.mark.parametrize("power", [-90, -101, -109, -117, -126])
@pytest.mark.parametrize("T", [50, 300, 3000])
def test_window_all_weigh_the_same(T, power):
    # of n equal values: n products, each rounded to 2^-149 with the sum at 2^-14 of it at least, beside the weights' 2^-16
    v = small(gen(2), (1, 1, 1, 64), power).expand(1, T, 1, 64)
    q = rnd(gen(3), (1, T, 1, 64), "bf16").to(DEV)
    o = f64(tk.window_attention(q, q, v.to(DEV), scale=0.0))
    assert (np.abs(o - f64(v)) <= (U["bf16"] + 2.0 ** -15 + T * 2.0 ** -24) * np.abs(f64(v)) + HALF_STEP + 2.0 ** -135).all()


@pytest.mark.parametrize("T,window,sinks", [(300, None, 0), (20000, None, 0), (9000, 3000, 70)])
@pytest.mark.parametrize("scale", [0.0, 0.1, 1.0])
def test_window_means_of_the_largest_values(T, window, sinks, scale):
    say("window large values", T, window, sinks, scale)
    top = float(torch.finfo(BF).max)
    q = rnd(gen(4), (1, T, 1, 64), "bf16").to(DEV)
    v = torch.full((1, T, 1, 64), top, device=DEV).to(BF)
    v[..., 32:] *= -1
    o = tk.window_attention(q, q, v, window, sinks, scale=scale)
    assert torch.isfinite(o).all() and bool((o == v).all())


@pytest.mark.parametrize("scale", [1.0, 1e3, 1e6, 1e8, 1e10, 3e15, 1e25])
@pytest.mark.parametrize("T", [40, 700])
def test_window_ties_of_large_scores_over_the_largest_values(T, scale):
    top = float(torch.finfo(BF).max)
    for D in (64, 128):
        x = torch.ones((2, T, 1, D), device=DEV, dtype=BF)
        v = torch.full_like(x, top)
        x[1, T // 3:] = 0.5  # the tokens in front are ahead by half the score
        o = tk.window_attention(torch.ones_like(x), x, v, scale=scale)
        assert bool((o == v).all())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("step", [3, 6, 8, 10, 12, 20])
@pytest.mark.parametrize("large", [10, 13, 15, 18])
def test_window_large_scores_that_rise_from_tile_to_tile(large, step, dt):
    # from 2^20 to 2^28, by `step` every 64 keys: fp32 scores there err by 2^4 at most (and by nothing at 2^20 or below)
    T = 1000
    q, k = torch.zeros((1, T, 1, 64)), torch.zeros((1, T, 1, 64))
    q[..., 0], k[..., 0] = 32.0, 32.0
    q[..., 1] = step * 2.0 ** -large if dt == "bf16" or large <= 13 else step * 2.0 ** -13
    k[..., 1] = (torch.arange(T) // 64).view(1, T, 1) * (1.0 if dt == "bf16" or large <= 13 else 2.0 ** (13 - large))
    v = rnd(gen(11), (1, T, 1, 64), dt).to(DEV)
    o = tk.window_attention(q.to(v.dtype).to(DEV), k.to(v.dtype).to(DEV), v, scale=2.0 ** large)
    top = float(v.float().abs().max())
    assert torch.isfinite(o).all() and float(o.float().abs().max()) <= top * (1 + 2 * U[dt])
    if step == 20 and large <= 15:  # what is a tile behind weighs exp(-20 + 2^2 ln 2) at most
        for i in range(64, T, 97):
            want = f64(v)[0, i // 64 * 64:i + 1].mean(0)
            assert np.abs(f64(o)[0, i] - want).max() <= (U[dt] + 2.0 ** -15 + 2 * 64 * np.exp(-17)) * top, i


@pytest.mark.parametrize("power", [-90, -105, -109, -112, -117, -120, -125, -126])
@pytest.mark.parametrize("n", [1, 40, 300, 3000, 20000])
def test_paged_one_token_has_all_the_weight(n, power):
    say("paged small", n, power)
    c = Cache(gen(5), 1, n, 16, 1, 64, 128, "bf16")
    q = torch.zeros((1, 2, 64), dtype=BF, device=DEV)
    q[..., 0] = 32.0
    c.v.copy_(small(gen(6), c.v.shape, power))
    for at in (0, n // 3, n - 1):
        c.k.zero_()
        page, row = int(c.table[0, at // 16]), at % 16
        c.k[page, row, 0, 0] = 16.0
        want = f64(c.v[page, row, 0])
        for mass in (None, torch.zeros((1, 1, c.columns), device=DEV)):
            o = f64(tk.paged_attention(q, c.k, c.v, c.table, i32([n]), scale=1.0, mass=mass))
            assert (np.abs(o - want) <= U["bf16"] * np.abs(want) + HALF_STEP + 2 * 2.0 ** -136).all(), at
        assert float(mass[0, 0, at]) == 2.0 and float(mass.sum()) == 2.0


@pytest.mark.parametrize("power", [-90, -109, -117, -126])
@pytest.mark.parametrize("n", [50, 3000, 20000])
def test_paged_all_weigh_the_same(n, power):
    c = Cache(gen(7), 1, n, 16, 1, 64, 64, "bf16")
    v = small(gen(8), (64,), power).to(DEV)
    c.v.copy_(v.expand_as(c.v))
    o = f64(tk.paged_attention(torch.ones((1, 2, 64), dtype=BF, device=DEV), c.k, c.v, c.table, i32([n]), scale=0.0))
    assert (np.abs(o - f64(v)) <= (U["bf16"] + 2.0 ** -15 + n * 2.0 ** -24) * np.abs(f64(v)) + HALF_STEP + 2.0 ** -135).all()


@pytest.mark.parametrize("n", [50, 3000, 20000, 130560])
@pytest.mark.parametrize("scale", [0.0, 0.1, 1.0])
def test_paged_means_of_the_largest_values(n, scale):
    top = float(torch.finfo(BF).max)
    for B in (1, 70):
        if B * n > 300000:
            continue
        c = Cache(gen(9), B, n, 64, 1, 64, 64, "bf16")
        c.v.fill_(top)
        c.v[..., 32:] *= -1
        o = tk.paged_attention(rnd(gen(10), (B, 2, 64), "bf16").to(DEV), c.k, c.v, c.table, i32([n] * B), scale=scale)
        assert bool((o == c.v[0, 0]).all())


def nearly_equal(B, dt):
    """Sequences of three tokens.  The third sees two whose weights differ by 2^-9 of them at most, with values 1 and -1,
    and itself, heavier and with a value of 0: (queries, keys, values)."""
    g = gen(12)
    q, k, v = (torch.zeros((B, 3, 1, 16)) for _ in range(3))
    q[:, 2, 0, 0], q[:, 2, 0, 1] = 0.7 * torch.rand(B, generator=g), 1.0
    k[:, :2, 0, 0], k[:, :2, 0, 1] = -1.0, 2.0 ** -9 * torch.rand((B, 2), generator=g)
    v[:, 0], v[:, 1] = 1.0, -1.0
    return [x.to(torch.float16 if dt == "fp16" else BF) for x in (q, k, v)]


@pytest.mark.parametrize("form", ["prompt", "token"])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_bits_of_a_weight(form, dt):
    # a weight's terms hold it to 2^-22 (fp16) and 2^-17 (bf16), its exponential and the sums to 2^-20 together; the
    # difference of the two, 2^-10 of them, is rounded
    B = 3000
    q, k, v = (x.to(DEV) for x in nearly_equal(B, dt))
    if form == "prompt":
        o = f64(tk.window_attention(q, k, v, scale=1.0))[:, 2, 0]
    else:
        x = torch.zeros((2, B, 4, 1, 16), dtype=q.dtype, device=DEV)
        x[0, :, :3], x[1, :, :3] = k, v
        o = f64(tk.paged_attention(q[:, 2], x[0], x[1], torch.arange(B, dtype=torch.int32, device=DEV)[:, None], i32([3] * B), scale=1.0))[:, 0]
    w = np.exp((f64(q)[:, 2:] * f64(k)).sum((2, 3)))
    w /= w.sum(1, keepdims=True)
    want = (w[:, 0] - w[:, 1])[:, None]
    bound = (2.0 ** (-22 if dt == "fp16" else -17) + 2.0 ** -20) * w[:, :2].sum(1)[:, None] + U[dt] * np.abs(want)
    assert (np.abs(o - want) <= bound).all(), float((np.abs(o - want) / bound).max())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("shift", [-2.0, 0.0, 2.0])
@pytest.mark.parametrize("d", [-4.0, -1.0, 1.0, 4.0])
def test_window_scores_around_the_border_of_large_ones(d, shift, dt):
    # two tiles of 64 keys, each of two waves' own, whose scores of 2^22 ln 2 and d more are taken for large or not; a score
    # there errs by a quarter of a power of two, for the rounded product, at most
    for sign in (1.0, -1.0):
        q, k, v = (torch.zeros((1, 128, 1, 16)) for _ in range(3))
        q[..., 0], q[..., 1], k[..., 0] = 32.0, 2.0 ** -5, 32.0
        scale = sign * (2.0 ** 22 * np.log(2) + shift) / 1024
        k[0, 64:, 0, 1] = d / scale * 32
        v[0, :64] = 1.0
        q, k, v = (x.to(torch.float16 if dt == "fp16" else BF).to(DEV) for x in (q, k, v))
        o = f64(tk.window_attention(q, k, v, scale=float(scale)))[0, 127, 0]
        delta = f64(k)[0, 127, 0, 1] * scale / 32
        assert (np.abs(np.log(o / (1 - o)) + delta) <= 0.5 * np.log(2) + 2 * U[dt] / min(o[0], 1 - o[0])).all(), (sign, o)
