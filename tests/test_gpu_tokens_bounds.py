"""Decay attention against the float64 oracle in tighter bounds than its formats' worst case.

The chunked form multiplies 16-bit operands.  Scores and states go in as two 16-bit terms, 2^-22 (fp16) or 2^-16
(bf16) of a value, which with the roundings of their weights (a few 2^-24) stays below 2^-20 and 2^-15 of the sum of
magnitudes; sums over the sequence are fp32.  What is left is the one rounding of the output.
"""
import numpy as np
import pytest
import torch

from oracle import tokens as ref
from paper_2502_20762_amd import tokens as tk
from test_gpu_tokens import DEV, DT, F32, TINY, U, check, f64, gen, rnd, say

pytestmark = pytest.mark.gpu

TERMS = {"fp16": 2.0 ** -20, "bf16": 2.0 ** -15}


def attend(q, k, v, ld, S0, scale, dt, what):
    """Runs the operator and holds its outputs to the bound; returns them, the state, and the oracle's (o, S, |o|, |S|)."""
    ld = torch.tensor(ld, dtype=torch.float32)
    o, S = tk.decay_attention(*(x.to(DEV) for x in (q, k, v)), ld.to(DEV), None if S0 is None else S0.to(DEV),
                              scale=scale, return_state=True)
    torch.cuda.synchronize()
    n = [f64(x) for x in (q, k, v)]
    s = None if S0 is None else f64(S0)
    want, wS = ref.decay_attention(*n, f64(ld), s, None, scale)
    mag, mS = ref.decay_attention(*(np.abs(x) for x in n), f64(ld), None if s is None else np.abs(s), None, scale)
    e = (TERMS[dt] + (q.shape[1] + 256) * F32) * mag
    check(o, want, e * (1 + U[dt]) + U[dt] * np.abs(want) + TINY[dt], what)
    return o, S, want, wS, mag, mS


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T,D,V", [(64, 64, 64), (50, 128, 32), (700, 64, 64), (300, 128, 128), (130, 40, 75)])
def test_outputs_err_as_their_rounding_does(T, D, V, dt):
    say("decay, one rounding", T, D, V, dt)
    g = gen(1)
    q, k = (rnd(g, (2, T, 2, D), dt) for _ in range(2))
    v = rnd(g, (2, T, 2, V), dt)
    S0 = torch.randn((2, 2, D, V), generator=g) * 4
    o, _, want, *_ = attend(q, k, v, (-0.02, -0.3), S0, D ** -0.5, dt, (T, D, V, dt))
    rounded = f64(torch.from_numpy(want).to(DT[dt]))
    # terms and sums are below a hundredth of the rounding, and their errors are apart from it
    assert ((f64(o) - want) ** 2).mean() <= 1.05 ** 2 * ((rounded - want) ** 2).mean(), (T, D, V, dt)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("quiet", [2.0 ** -8, 2.0 ** -16])
def test_quiet_queries_beside_loud_ones(quiet, dt):
    say("decay, quiet queries", quiet, dt)
    g = gen(2)
    q, k, v = (torch.randn((1, 200, 2, 64), generator=g) for _ in range(3))
    q[:, 1::2] *= quiet
    S0 = torch.randn((1, 2, 64, 64), generator=g)
    attend(*(x.to(DT[dt]) for x in (q, k, v)), (-0.02, -0.3), S0, 64.0, dt, (quiet, dt))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("loud", [40, 100])
def test_quiet_keys_after_loud_ones_that_have_decayed(loud, dt):
    # the loud keys' weights are below 2^-57 from twenty tokens on
    say("decay, quiet keys", loud, dt)
    g = gen(3)
    q, k, v = (torch.randn((1, 250, 2, 64), generator=g) for _ in range(3))
    k *= 2.0 ** -9
    k[:, loud - 10:loud] *= 2.0 ** 18
    attend(*(x.to(DT[dt]) for x in (q, k, v)), (-2.0, -2.5), None, 1.0, dt, (loud, dt))


def state_check(S, wS, mS, T, what):
    # terms to 2^-22 of a weighted value, their weights to a few 2^-24, fp32 sums
    check(S, wS, ((T + 16) * F32 + 2.0 ** -21) * mS + 1e-37, (what, "state"))


@pytest.mark.parametrize("T", [3, 64, 150, 700])
@pytest.mark.parametrize("quiet", [2.0 ** -12, 2.0 ** -16, 2.0 ** -20])
def test_quiet_columns_keep_the_bits_of_the_state(quiet, T):
    # columns of very different magnitude in one head: each as exact as if it were alone
    say("decay, quiet columns", quiet, T)
    g = gen(4)
    q, k, v = (torch.randn((1, T, 2, 64), generator=g) for _ in range(3))
    v[..., 1::2] *= quiet
    v *= 2.0 ** 6
    o, S, want, wS, mag, mS = attend(*(x.half() for x in (q, k, v)), (-0.02, -0.3), None, 1.0, "fp16", (quiet, T))
    state_check(S, wS, mS, T, (quiet, T))


@pytest.mark.parametrize("loud", [5, 40, 100])
def test_quiet_values_after_loud_ones_that_have_decayed_keep_the_bits_of_the_state(loud):
    say("decay, quiet values", loud)
    g = gen(5)
    q, k, v = (torch.randn((1, 128, 2, 64), generator=g) for _ in range(3))
    v *= 2.0 ** -9
    v[:, loud - 5:loud] *= 2.0 ** 20
    q, k, v = (x.half() for x in (q, k, v))
    ld = torch.tensor([-2.0, -1.5])
    # the state alone: the loud tokens' own outputs are beyond fp16
    _, S = tk.decay_attention(*(x.to(DEV) for x in (q, k, v)), ld.to(DEV), return_state=True)
    _, wS = ref.decay_attention(f64(q), f64(k), f64(v), f64(ld))
    _, mS = ref.decay_attention(f64(q), np.abs(f64(k)), np.abs(f64(v)), f64(ld))
    state_check(S, wS, mS, 128, loud)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T", [3, 70, 400])
def test_a_state_near_the_end_of_fp32_stays_finite(T, dt):
    # magnitudes to 3.2e38 (2^127.9) in, a scale that brings the outputs back to ordinary numbers
    say("decay, large state", T, dt)
    g = gen(6)
    q, k, v = (torch.randn((1, T, 2, 64), generator=g) for _ in range(3))
    S0 = (torch.rand((1, 2, 64, 64), generator=g) * 2 - 1) * 3.2e38
    q *= 2.0 ** -8
    o, S, want, wS, mag, mS = attend(*(x.to(DT[dt]) for x in (q, k, v)), (0.0, -0.01), S0, 2.0 ** -120, dt, (T, dt))
    state_check(S, wS, mS, T, (T, dt))


@pytest.mark.parametrize("T", [3, 70, 400])
def test_a_state_past_the_largest_bf16_stays_finite(T):
    # fp32 ends at 3.4028e38, bf16 at 3.3895e38: between them a first term must not round up
    say("decay, state past bf16", T)
    g = gen(7)
    q, k, v = (torch.randn((1, T, 2, 64), generator=g) for _ in range(3))
    S0 = torch.where(torch.rand((1, 2, 64, 64), generator=g) < 0.5, -3.402e38, 3.402e38)
    k *= 2.0 ** -8  # so that what is added is far from what a state at the end still holds
    q *= 2.0 ** -8
    o, S, want, wS, mag, mS = attend(*(x.bfloat16() for x in (q, k, v)), (0.0, -0.01), S0, 2.0 ** -120, "bf16", T)
    state_check(S, wS, mS, T, T)
