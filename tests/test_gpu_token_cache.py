"""The cache of a batch of streams: what it holds and lets go of, against lists of tokens kept on the host."""
import pytest
import torch

from attention_util import DEV
from paper_2502_20762_amd.mixer import TokenCache

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
