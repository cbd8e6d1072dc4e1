"""The reference of the token operators against independent forms: closed forms, other orders of the same sums."""
import math

import numpy as np
import pytest

from oracle import tokens as tk


def test_activations_closed_forms():
    v = np.linspace(-9, 9, 181)
    assert np.allclose(tk.ACTIVATIONS["silu"](v), v / (1 + np.exp(-v)), rtol=1e-13, atol=0)
    assert np.allclose(tk.ACTIVATIONS["wsilu"](v), v / (1 + np.exp(-4 * v)), rtol=1e-9, atol=1e-18)
    phi = np.array([0.5 * math.erfc(-a / math.sqrt(2)) for a in v])
    assert np.allclose(tk.ACTIVATIONS["gelu"](v), v * phi, rtol=1e-12, atol=1e-20)
    assert tk.ACTIVATIONS["lrelu"](np.array([-2.0, 3.0])).tolist() == [-0.2, 3.0]


def test_linear_by_loops():
    rng = np.random.default_rng(0)
    x, w, b, r = rng.standard_normal((3, 5)), rng.standard_normal((8, 5)), rng.standard_normal(8), rng.standard_normal((3, 4))
    got = tk.linear(x, w, b, r, "silu", gated=True)
    for i in range(3):
        for j in range(4):
            a = sum(x[i, c] * w[j, c] for c in range(5)) + b[j]
            g = sum(x[i, c] * w[j + 4, c] for c in range(5)) + b[j + 4]
            assert math.isclose(got[i, j], a / (1 + math.exp(-a)) * g + r[i, j], rel_tol=1e-12, abs_tol=1e-13)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_depends_on_the_difference_of_positions(interleaved):
    rng = np.random.default_rng(1)
    sections, D = (3, 2, 4), 20
    freq = rng.uniform(0.01, 1, 9)
    q, k = rng.standard_normal((1, 2, D)), rng.standard_normal((1, 2, D))

    def score(pq, pk):
        a = tk.norm_rope(q, None, np.array([pq]), freq, sections, interleaved=interleaved)
        b = tk.norm_rope(k, None, np.array([pk]), freq, sections, interleaved=interleaved)
        assert np.allclose((a * a).sum(-1), D, rtol=1e-5)  # the norm makes the mean square one, the rotation keeps it
        return (a * b).sum(-1)

    assert np.allclose(score((5, 9, 2), (1, 3, 8)), score((104, 6, 12), (100, 0, 18)), rtol=1e-11)


def test_zero_position_and_zero_head():
    x = np.zeros((2, 1, 8))
    x[1] = np.arange(8)
    y = tk.norm_rope(x, None, np.zeros((2, 1)), np.ones(4), (4,), eps=1e-6)
    assert np.all(y[0] == 0) and np.allclose(y[1], x[1] / np.sqrt((x[1] ** 2).mean() + 1e-6))


def test_decay_attention_as_a_masked_product():
    rng = np.random.default_rng(2)
    B, T, H, K, D, V = 2, 11, 4, 2, 3, 5
    q, k, v = rng.standard_normal((B, T, H, D)), rng.standard_normal((B, T, K, D)), rng.standard_normal((B, T, K, V))
    ld = np.array([-0.1, 0.0, -2.0, -np.inf])
    S0 = rng.standard_normal((B, H, D, V))
    lengths = np.array([11, 6])
    o, S = tk.decay_attention(q, k, v, ld, S0, lengths, scale=0.7)
    for b in range(B):
        n = lengths[b]
        for h in range(H):
            lam, kh = math.exp(ld[h]), h // 2
            D_ = np.array([[lam ** (i - j) if j <= i else 0.0 for j in range(n)] for i in range(n)])
            P = (q[b, :n, h] @ k[b, :n, kh].T) * D_
            ref = P @ v[b, :n, kh] + np.array([lam ** (i + 1) for i in range(n)])[:, None] * (q[b, :n, h] @ S0[b, h])
            assert np.allclose(o[b, :n, h], 0.7 * ref, rtol=1e-11, atol=1e-12)
            W = np.array([lam ** (n - 1 - j) for j in range(n)])
            assert np.allclose(S[b, h], lam ** n * S0[b, h] + (k[b, :n, kh] * W[:, None]).T @ v[b, :n, kh], rtol=1e-11,
                               atol=1e-12)
        assert np.all(o[b, n:] == 0)
