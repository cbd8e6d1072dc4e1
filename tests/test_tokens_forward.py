"""The token operators have no derivatives: a tensor with a forward-mode tangent is refused, whichever operand it is."""
import pytest
import torch
import torch.autograd.forward_ad as forward

from paper_2502_20762_amd import tokens as tk


def test_first_operands_before_anything_else():
    x = torch.ones((2, 8), dtype=torch.float16)
    with forward.dual_level():
        d = forward.make_dual(x, x)
        for call in (lambda: tk.linear(d, x), lambda: tk.qk_norm_rope(d, x), lambda: tk.decay_attention(d, x, x, x),
                     lambda: tk.window_attention(d, x, x), lambda: tk.paged_attention(d, x, x, x, x),
                     lambda: tk.cache_append(d, x, x, x, x, x), lambda: tk.cache_evict(d, x, x, x, x, 1, x)):
            with pytest.raises(ValueError, match="forward-mode"):
                call()
        with pytest.raises(ValueError, match="on the GPU"):
            tk.linear(x, x)


def calls():
    """(function, operands), each fit for a call."""
    def ones(*shape, dtype=torch.float16):
        return torch.ones(shape, dtype=dtype, device="cuda:0")

    i = torch.ones(1, dtype=torch.int32, device="cuda:0")
    table, more = i.view(1, 1) - 1, i.view(1, 1)
    q, k, v, kc, vc = ones(1, 4, 2, 16), ones(1, 4, 1, 16), ones(1, 4, 1, 16), ones(2, 4, 1, 16), ones(2, 4, 1, 16)
    mass = ones(1, 1, 4, dtype=torch.float32)
    return [(lambda x, w, b, r: tk.linear(x, w, b, r), (ones(3, 8), ones(5, 8), ones(5), ones(3, 5))),
            (lambda x, y, a, b: tk.qk_norm_rope(x, y, a, b), (q[0], k[0], ones(16), ones(16))),
            (lambda x, y, z, d, s: tk.decay_attention(x, y, z, d, s), (q, k, v, -ones(2, dtype=torch.float32), ones(1, 2, 16, 16, dtype=torch.float32))),
            (lambda x, y, z: tk.window_attention(x, y, z), (q, k, v)),
            (lambda x, y, z, m: tk.paged_attention(x, y, z, table, i, mass=m), (q[:, 0], kc, vc, mass)),
            (lambda x, y, a, b, m: tk.cache_append(x, y, a, b, table, i, mass=m), (k[:, :1], v[:, :1], kc, vc, mass)),
            (lambda a, b, m: tk.cache_evict(a, b, table, i, m, 1, more), (kc, vc, mass))]


@pytest.mark.gpu
def test_every_operand():
    for fn, operands in calls():
        fn(*operands)
        with forward.dual_level():
            fn(*operands)
            for n in range(len(operands)):
                dual = [forward.make_dual(t, torch.ones_like(t)) if j == n else t for j, t in enumerate(operands)]
                with pytest.raises(ValueError, match="forward-mode"):
                    fn(*dual)
                with torch.no_grad(), pytest.raises(ValueError, match="forward-mode"):
                    fn(*dual)
        fn(*operands)
