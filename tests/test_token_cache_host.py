"""The cache of a batch of streams, host side: what its constructor refuses."""
import pytest

from paper_2502_20762_amd.mixer import TokenCache


@pytest.mark.parametrize("bad", [dict(keep=8, sinks=3, recent=6), dict(keep=8, sinks=9), dict(keep=8, recent=9),
                                 dict(keep=8, sinks=-1), dict(keep=8, recent=-2, sinks=4), dict(keep=0), dict(keep=64),
                                 dict(keep=-3)])
def test_budgets_that_do_not_hold_what_they_fix(bad):
    with pytest.raises(ValueError):
        TokenCache(1, 64, 1, 8, device="cpu", **bad)


@pytest.mark.parametrize("good", [dict(), dict(keep=8, sinks=3, recent=5), dict(keep=1), dict(keep=63, sinks=63)])
def test_budgets_that_do(good):
    assert TokenCache(1, 64, 1, 8, device="cpu", **good).most == 0


def test_a_cache_without_a_budget_is_not_cut():
    with pytest.raises(ValueError, match="keep"):
        TokenCache(1, 64, 1, 8, device="cpu").evict()
