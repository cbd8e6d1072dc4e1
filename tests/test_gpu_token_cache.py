"""The cache of a batch of streams: what it holds and lets go of, against lists of tokens kept on the host."""
import numpy as np
import pytest
import torch

from attention_util import DEV, F32, f64, gen, rnd, weight_error
from paper_2502_20762_amd.mixer import CacheMixer, TokenCache
from paper_2502_20762_amd.tokens import grid_positions
from test_gpu_mixer import U, rms

pytestmark = pytest.mark.gpu


class Streams:
    """A cache whose tokens carry their number, and what each of its streams should hold."""

    def __init__(self, batch, capacity, **kw):
        self.cache = TokenCache(batch, capacity, 1, 8, page_size=4, device=DEV, **kw)
        self.held, self.next = [[] for _ in range(batch)], 1

    def append(self, counts, width=None, given=True):
        T = max(counts) if width is None else width
        x = torch.zeros((len(counts), T, 1, 8), dtype=torch.float16, device=DEV)
        for b, n in enumerate(counts):
            x[b, :n, 0, 0] = torch.arange(self.next, self.next + n)
        self.cache.append(x, -x, torch.tensor(counts, dtype=torch.int32, device=DEV) if given else None)
        for b, n in enumerate(counts):
            self.held[b] += range(self.next, self.next + n)
        self.next += T

    def check(self):
        c = self.cache
        assert c.lengths.tolist() == [len(h) for h in self.held] and c.most >= max(map(len, self.held))
        for b, h in enumerate(self.held):
            j = torch.arange(len(h), device=DEV)
            p = c.table[b, j // 4].long()
            assert c.k[p, j % 4, 0, 0].tolist() == h and c.v[p, j % 4, 0, 0].tolist() == [-x for x in h]


def test_appends_in_turn_fill_every_stream():
    s = Streams(2, 12)
    for t in range(24):
        s.append([t % 2, 1 - t % 2])
        s.check()
    for counts in ([1, 0], [0, 1], [1, 1]):
        with pytest.raises(ValueError, match="fit"):
            s.append(counts)
        s.check()
    for _ in range(20):
        s.append([0, 0], width=3)  # nothing always fits
    s.check()


def test_an_append_fits_by_its_counts_and_not_by_its_width():
    s = Streams(3, 20)
    s.append([15, 0, 3], width=15)
    s.append([5, 8, 0], width=9)
    s.check()
    with pytest.raises(ValueError, match="fit"):
        s.append([1, 0, 0], width=2)
    s.append([0, 12, 17], width=17)
    s.check()
    assert s.cache.most == 20


def test_a_long_prompt_of_short_streams_leaves_room():
    s = Streams(2, 100)
    s.append([10, 4], width=80)
    s.append([30, 30], given=False)
    s.check()
    s.append([60, 60], given=False)
    s.check()
    with pytest.raises(ValueError, match="fit"):
        s.append([1, 1], given=False)


def test_nothing_is_let_go_before_a_stream_would_overflow():
    s = Streams(2, 16, keep=6, sinks=2, recent=4)
    for t in range(24):  # 12 tokens of each
        s.append([t % 2, 1 - t % 2])
        s.check()
    s.append([4, 0], width=4)
    s.check()
    s.append([1, 0])  # the first stream overflows: all are cut back
    s.held = [h[:2] + h[len(h) - 4:] for h in (s.held[0][:-1], s.held[1])]
    s.held[0].append(s.next - 1)
    s.check()
    assert s.cache.most == 7


def test_an_eviction_makes_room_for_counts():
    s = Streams(2, 10, keep=6, sinks=1, recent=5)
    s.append([9, 2])
    with pytest.raises(ValueError, match="fit"):
        s.append([5, 0])
    s.check()
    s.append([4, 8], width=9)  # 6 + 4 and 2 + 8, of a width that would not fit
    s.held[0] = s.held[0][:1] + s.held[0][4:]
    s.check()
    assert s.cache.most == 10


def test_streams_of_the_same_length_are_counted_on_the_host():
    s = Streams(2, 64, keep=6, sinks=2, recent=4)
    for t in range(40):
        s.append([3, 3], given=False)
        assert s.cache.most == int(s.cache.lengths.max()) and s.cache.exact


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("B,T,H,K,window,sinks,counts", [
    (1, 150, 4, 2, None, 0, None), (1, 64, 2, 2, 30, 3, None), (3, 70, 4, 1, None, 0, [70, 0, 33]),
    (70, 9, 2, 1, None, 0, [b % 11 - 1 for b in range(70)]), (2, 1, 2, 2, None, 0, None)])
def test_a_prompt_weighs_what_its_tokens_one_by_one_do(B, T, H, K, window, sinks, counts, dt):
    # the same weights, each by its error twice, summed in another order
    g, D, keep, more = gen(5), 64, max(1, T // 2), 40
    q, k, v = (rnd(g, (B, T + more, h, D), dt).to(DEV) for h in (H, K, K))
    n = torch.full((B,), T) if counts is None else torch.tensor(counts).clamp(0, T)
    a, b = (TokenCache(B, T + 8, K, D, keep=keep, sinks=min(2, keep), dtype=q.dtype, device=DEV) for _ in range(2))
    given = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
    a.append(k[:, :T], v[:, :T], given)
    a.weigh_prompt(q[:, :T], given, window, sinks)
    for t in range(T):
        one = (t < n).to(torch.int32).to(DEV)
        before = b.mass.clone()
        b.append(k[:, t:t + 1], v[:, t:t + 1], one)
        b.attend(q[:, t], window, sinks)
        b.mass = torch.where(one[:, None, None] > 0, b.mass, before)  # a stream that got nothing asks nothing
    assert torch.equal(a.lengths, b.lengths) and a.lengths.tolist() == n.tolist()
    e = 2 * 2 * weight_error(f64(q), f64(k), D ** -0.5, D, "fp16") + 4 * T * F32
    assert ((a.mass - b.mass).abs() <= e * b.mass).all()
    assert np.abs(f64(a.mass.sum((1, 2))) - H * f64(n)).max() <= 1e-3 * H * T
    # and both keep the same tokens at the evictions that follow
    for t in range(T, T + more):
        for c in (a, b):
            c.append(k[:, t:t + 1], v[:, t:t + 1])
        x, y = a.attend(q[:, t], window, sinks), b.attend(q[:, t], window, sinks)
        assert torch.equal(x, y) and torch.equal(a.lengths, b.lengths), t


def test_a_prompt_and_steps_keep_what_steps_alone_keep():
    m = CacheMixer(64, heads=4, kv_heads=2, sinks=3, device=DEV)
    x = torch.randn((60, 64), generator=gen(6)).half().to(DEV)
    pos = grid_positions(1, 6, 10, device=DEV)
    a, b = (m.new_cache(64, keep=40, recent=8) for _ in range(2))
    m(x[None], pos, a)
    for t in range(60):
        m.step(x[t:t + 1], pos[t:t + 1], b)
    # queries and keys were rounded after products in another order
    assert rms(a.mass, f64(b.mass)) <= 16 * U[torch.float16]
    heavy = a.mass[0, :, 3:52].topk(29, 1).indices.sort(1).values
    kept = a.evict()
    assert torch.equal(kept[0, :, 3:32].long(), heavy + 3)


def test_a_prompt_without_a_budget_weighs_nothing():
    m = CacheMixer(64, window=9, device=DEV)
    cache = m.new_cache(40)
    m(torch.randn((1, 30, 64), device=DEV).half(), grid_positions(1, 5, 6, device=DEV), cache)
    assert bool((cache.mass == 0).all())
    cache = CacheMixer(64, device=DEV).new_cache(40)
    cache.weigh_prompt(torch.ones((1, 30, 4, 64), dtype=torch.float16, device=DEV))
    assert cache.mass is None


def test_a_refused_append_lets_go_of_nothing():
    s = Streams(2, 12, keep=6, sinks=2, recent=2)
    s.append([10, 10], given=False)
    c = s.cache
    x, two = torch.ones((2, 4, 1, 8), dtype=torch.float16, device=DEV), torch.tensor([2, 1], dtype=torch.int32, device=DEV)
    mass = c.mass.clone()
    for bad in ((x.bfloat16(), x.bfloat16()), (x, x.float()), (x[..., :7], x), (x.expand(2, 4, 3, 8), x), (x, x[:, :3]),
                (x[:1], x[:1]), (x.cpu(), x), (x, x, two.long()), (x, x, two[:1]), (x, x, two.float()), (x, x, two.cpu()),
                (x, x[..., ::2]), (c.k[:2, :4], x), (x, c.v[:2, :4]), (x.clone().requires_grad_(), x)):
        table, most = c.table, c.most
        with pytest.raises((ValueError, RuntimeError)):
            c.append(*bad)
        assert c.table is table and c.most == most and c.lengths.tolist() == [10, 10] and torch.equal(c.mass, mass)
        s.check()
    s.append([4, 4], given=False)
    assert c.lengths.tolist() == [10, 10] and c.most == 10
