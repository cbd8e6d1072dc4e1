"""Windows, sinks and recent tokens that no field of the library holds: refused, not cut to their lower 64 bits."""
import pytest
import torch

from attention_util import DEV, Cache, gen
from paper_2502_20762_amd import ncodec as nc
from paper_2502_20762_amd import tokens as tk
from test_gpu_paged import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1 << 63, 1 << 64, (1 << 64) + 3, 10 ** 30])
def test_more_than_64_bits(n):
    x = torch.ones((1, 4, 2, 64), dtype=torch.float16, device=DEV)
    c = Cache(gen(1), 2, 64, 16, 2, 64, 64, "fp16")
    mass, ln, q = torch.zeros((2, 2, 64), device=DEV), i32([3, 4]), torch.ones((2, 4, 64), dtype=torch.float16, device=DEV)
    k = c.k.clone()
    for bad in (lambda: tk.window_attention(x, x, x, n), lambda: tk.window_attention(x, x, x, None, n),
                lambda: tk.window_attention(x, x, x, None, -n), lambda: tk.paged_attention(q, c.k, c.v, c.table, ln, n),
                lambda: tk.paged_attention(q, c.k, c.v, c.table, ln, 2, n),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, mass, 5, c.table.clone(), n),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, mass, 5, c.table.clone(), 0, n),
                lambda: tk.cache_evict(c.k, c.v, c.table, ln, mass, n, c.table.clone())):
        with pytest.raises((ValueError, nc.NcodecError)):
            bad()
    assert torch.equal(k, c.k)
