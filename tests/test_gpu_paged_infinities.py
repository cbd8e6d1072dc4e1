"""One token over a cache whose seen positions all have scores of -inf: no weight is a number, wherever they lie in a step
of 32 positions."""
import pytest
import torch

from attention_util import DEV, Cache, gen, rnd
from paper_2502_20762_amd import tokens as tk
from test_gpu_paged import INF, i32

pytestmark = pytest.mark.gpu


def seen_of(n, window, sinks):
    j = torch.arange(n)
    return (j >= n - window) | (j < sinks) if window else j >= 0


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("page", [1, 8, 16, 32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 0), (5, 0), (1, 1), (3, 7)])
def test_all_that_a_window_shows(window, sinks, page, dt):
    g = gen(1)
    for n in (1, 2, 4, 5, 6, 8, 9, 12, 13, 16, 17, 20, 21, 24, 28, 31, 32, 33, 37, 48, 70):
        c = Cache(g, 2, n + 40, page, 1, 64, 64, dt)
        q, seen = torch.ones((2, 3, 64), dtype=c.k.dtype, device=DEV), seen_of(n, window, sinks).to(DEV)
        for j in seen.nonzero().flatten().tolist():  # of the first sequence; the second has numbers
            c.k[int(c.table[0, j // page]), j % page] = -INF
        mass = torch.ones((2, 1, c.columns), device=DEV)
        o = tk.paged_attention(q, c.k, c.v, c.table, i32([n, n]), window, sinks, mass=mass)
        assert torch.isnan(o[0]).all() and torch.isfinite(o[1]).all(), n
        assert torch.isnan(mass[0, 0, :n][seen]).all() and bool((mass[0, 0, :n][~seen] == 1).all()), n
        assert bool((mass[0, 0, n:] == 1).all()) and torch.isfinite(mass[1]).all(), n
        # as the prompt form has it
        k, v = (x[c.table[0, torch.arange(n) // page].long(), torch.arange(n, device=DEV) % page][None] for x in (c.k, c.v))
        assert torch.isnan(tk.window_attention(q[:1, None].expand(1, n, 3, 64), k, v, window, sinks)[0, -1]).all(), n


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("n", [30, 3000])
@pytest.mark.parametrize("at", [0, 1, 3, 5, 6, 7])
def test_all_that_has_a_page(at, n, dt):
    # one page of four tokens is there: alone in its step, its wave's share and, of 3,000 tokens, its workgroup's
    c = Cache(gen(2), 1, n, 4, 1, 64, 64, dt)
    column = (0 if n == 30 else 400) + at
    table = torch.full_like(c.table, -1)
    table[0, column] = c.table[0, column]
    c.k.fill_(-INF)
    mass = torch.zeros((1, 1, c.columns), device=DEV)
    q = rnd(gen(3), (1, 2, 64), dt).abs().to(DEV)
    for m in (None, mass):
        assert torch.isnan(tk.paged_attention(q, c.k, c.v, table, i32([n]), mass=m)).all()
    there = slice(4 * column, min(4 * column + 4, n))
    assert torch.isnan(mass[0, 0, there]).all()
    mass[0, 0, there] = 0
    assert bool((mass == 0).all())
