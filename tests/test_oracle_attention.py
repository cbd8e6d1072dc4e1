"""The reference of the softmax attentions and of the cache's upkeep against independent forms."""
import numpy as np
import pytest

from oracle import tokens as tk


@pytest.mark.parametrize("window,sinks", [(None, 0), (1, 0), (4, 0), (4, 2), (3, 50), (50, 2)])
def test_window_attention_as_a_masked_product(window, sinks):
    rng = np.random.default_rng(0)
    B, T, H, K, D, V = 2, 13, 4, 2, 3, 5
    q, k, v = rng.standard_normal((B, T, H, D)), rng.standard_normal((B, T, K, D)), rng.standard_normal((B, T, K, V))
    lengths = [13, 6]
    o = tk.window_attention(q, k, v, window, sinks, lengths, 0.7)
    i, j = np.indices((T, T))
    mask = (j <= i) & ((j < sinks) | (i - j < (window or T)))
    z = 0.7 * np.einsum("bihd,bjhd->bhij", q, np.repeat(k, 2, 2))
    w = np.where(mask, np.exp(z), 0.0)
    want = np.einsum("bhij,bjhv->bihv", w / w.sum(-1, keepdims=True), np.repeat(v, 2, 2))
    want[1, 6:] = 0
    assert np.allclose(o, want, rtol=1e-12, atol=1e-13)


def test_one_token_over_pages_is_the_last_of_a_prompt_and_weights_sum_to_one():
    rng = np.random.default_rng(1)
    B, T, H, K, D, V, page = 3, 21, 4, 2, 3, 5, 4
    q, k, v = rng.standard_normal((B, T, H, D)), rng.standard_normal((B, T, K, D)), rng.standard_normal((B, T, K, V))
    table = rng.permutation(20)[:18].reshape(B, 6)
    kc, vc = np.zeros((20, page, K, D)), np.zeros((20, page, K, V))
    kc, vc, mass = tk.cache_append(k, v, kc, vc, table, [0] * B, None, np.ones((B, K, 24)))
    assert (mass[..., :T] == 0).all() and (mass[..., T:] == 1).all()
    for window, sinks in ((None, 0), (5, 3)):
        o, m = tk.paged_attention(q[:, -1], kc, vc, table, [T] * B, window, sinks, 0.7, mass * 0)
        assert np.allclose(o, tk.window_attention(q, k, v, window, sinks, None, 0.7)[:, -1], rtol=1e-12, atol=1e-13)
        assert np.allclose(m.sum(-1), H // K) and np.count_nonzero(m[0, 0]) == len(tk.seen(T - 1, window, sinks))
    o, _ = tk.paged_attention(q[:, 0], kc, vc, table, [0, 1, -1], None, 0)
    assert (o[0] == 0).all() and (o[2] == 0).all() and np.allclose(o[1], v[1, 0].repeat(2, 0))
    # a number that is no page holds nothing
    table2 = table.copy()
    table2[:, 0] = (-1, 20, 1 << 30)
    a, _ = tk.paged_attention(q[:, -1], kc, vc, table2, [T] * B, None, 0)
    b, _ = tk.paged_attention(q[:, -1], kc, vc, table, [T] * B, T - page, 0)
    assert np.allclose(a, b)


def test_evict_by_hand():
    page, K = 2, 1
    kc = np.arange(24.0).reshape(12, page, K, 1)
    vc = -kc
    table, new = np.array([[4, 0, 2, 1]]), np.array([[7, 9]])
    mass = np.array([[[9.0, 1.0, np.nan, 3.0, 3.0, -0.0, 0.0, 2.0]]])
    k2, v2, n, m, kept = tk.cache_evict(kc, vc, table, [8], mass, 4, new)
    assert kept.tolist() == [[[0, 2, 3, 4]]] and n.tolist() == [4] and np.isnan(m[0, 0, 1])
    assert k2[7, :, 0, 0].tolist() == [8, 0] and k2[9, :, 0, 0].tolist() == [1, 4] and (v2 == -k2).all()
    assert (np.delete(k2, [7, 9], 0) == np.delete(kc, [7, 9], 0)).all()
    assert tk.cache_evict(kc, vc, table, [8], mass, 3, new)[4].tolist() == [[[0, 2, 3]]]  # of equals the earlier
    assert tk.cache_evict(kc, vc, table, [8], mass, 4, new, 2, 2)[4].tolist() == [[[0, 1, 6, 7]]]
    assert tk.cache_evict(kc, vc, table, [8], mass, 3, new, 1, 1)[4].tolist() == [[[0, 2, 7]]]
    k2, _, n, m, kept = tk.cache_evict(kc, vc, table, [3], mass, 4, new)
    assert kept.tolist() == [[[0, 1, 2, -1]]] and n.tolist() == [3] and m[0, 0, 3] == 0 and k2[9, 1, 0, 0] == kc[9, 1, 0, 0]
    mass[0, 0, :] = [0.0, -0.0, 0.0, -0.0, -1.0, np.inf, -np.inf, -2.0]
    assert tk.cache_evict(kc, vc, table, [8], mass, 4, new)[4].tolist() == [[[0, 1, 2, 5]]]
