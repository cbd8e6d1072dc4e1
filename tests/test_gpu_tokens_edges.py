"""Token operators at the edges of their arguments: values that are no numbers, infinities, and what is refused."""
import numpy as np
import pytest
import torch

from oracle import tokens as ref
from paper_2502_20762_amd import ncodec as nc
from paper_2502_20762_amd import tokens as tk
from test_gpu_tokens import DEV, DT, f64, gen, rnd, say

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


# few rows, and tiles: more than 2^19 products of rows and weight rows, loaded directly and (k odd) through registers
@pytest.mark.parametrize("m,k,n", [(5, 70, 90), (300, 256, 256), (700, 512, 1024), (700, 77, 1024)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "lrelu", "wsilu", "silu", "gelu"])
def test_nan_goes_through_every_activation(act, gated, m, k, n):
    say("nan", act, gated, m, k, n)
    g = gen(1)
    rows = 2 * n if gated else n
    for dt in ("fp16", "bf16"):
        x, w, b = rnd(g, (m, k), dt), rnd(g, (rows, k), dt, k ** -0.5), rnd(g, (rows,), dt)
        clean = tk.linear(x.to(DEV), w.to(DEV), b.to(DEV), act=act, gated=gated).cpu()
        assert torch.isfinite(clean).all()
        x[1, 3], w[2, k - 1], b[rows - 1] = NAN, NAN, NAN  # a row, a feature, a feature
        y = tk.linear(x.to(DEV), w.to(DEV), b.to(DEV), act=act, gated=gated).cpu()
        hit = torch.zeros((m, n), dtype=torch.bool)
        hit[1] = hit[:, 2] = hit[:, n - 1] = True
        assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], clean[~hit]), dt


@pytest.mark.parametrize("m,n", [(6, 40), (800, 1024)])
def test_gelu_of_infinities(m, n):
    # v Phi(v) ends at 0 and at infinity
    x = torch.zeros((m, 8), dtype=torch.float16, device=DEV)
    x[0, 0], x[1, 0] = INF, -INF
    w = torch.ones((n, 8), dtype=torch.float16, device=DEV)
    y = tk.linear(x, w, act="gelu")
    assert bool((y[0] == INF).all()) and bool((y[1:] == 0).all())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 90, 700])
def test_a_decay_that_is_no_number_is_not_taken_for_one(T, dt):
    # its head has no outputs and no state, the other heads have theirs; without tokens the state stands still
    say("nan decay", T, dt)
    g = gen(2)
    q, k, v = (rnd(g, (3, T, 3, 64), dt).to(DEV) for _ in range(3))
    S0 = torch.randn((3, 3, 64, 64), generator=g).to(DEV)
    lengths = torch.tensor([T, T - T // 3, 0], dtype=torch.int32, device=DEV)
    ld = torch.tensor([-0.1, -0.02, -0.3], device=DEV)
    o, S = tk.decay_attention(q, k, v, ld, S0, lengths, return_state=True)
    ld[1] = NAN
    o2, S2 = tk.decay_attention(q, k, v, ld, S0, lengths, return_state=True)
    for b, n in enumerate(lengths.tolist()):
        assert torch.isnan(o2[b, :n, 1]).all() and bool((o2[b, n:, 1] == 0).all())
        assert torch.isnan(S2[b, 1]).all() if n else torch.equal(S2[b, 1], S0[b, 1])
    for h in (0, 2):
        assert torch.equal(o2[:, :, h], o[:, :, h]) and torch.equal(S2[:, h], S[:, h])


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 6, 70, 700])
def test_state_without_tokens_stands_still_whatever_it_holds(T, dt):
    g = gen(3)
    q, k, v = (rnd(g, (2, T, 2, 64), dt).to(DEV) for _ in range(3))
    S0 = torch.randn((2, 2, 64, 64), generator=g).to(DEV)
    S0[0, 0, 1, 2], S0[0, 1, 60, 63], S0[0, 1, 3, 4] = INF, -INF, 3.0e38
    lengths = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    for decay in (0.0, -0.5):
        ld = torch.full((2,), decay, device=DEV)
        o, S = tk.decay_attention(q, k, v, ld, S0, lengths, return_state=True)
        assert torch.equal(S[0], S0[0]) and bool((o[0] == 0).all()) and torch.isfinite(S[1]).all()


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("T", [4, 100, 400])
@pytest.mark.parametrize("where", ["q", "k", "v", "state"])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
def test_what_is_not_finite_reaches_what_the_formula_says(what, where, T, dt):
    # one value, in the middle of its stretch: the outputs and the state's elements that are not finite are the oracle's
    say("not finite", what, where, T, dt)
    g = gen(4)
    x = {name: rnd(g, (1, T, 2, 64), dt) for name in "qkv"}
    x["state"] = torch.randn((1, 2, 64, 64), generator=g)
    at = (0, 1, 5, 40) if where == "state" else (0, T // 2, 1, 40)
    x[where][at] = what
    for decay in (-0.05, 0.0):
        ld = torch.tensor([-0.1, decay])
        o, S = tk.decay_attention(*(x[name].to(DEV) for name in "qkv"), ld.to(DEV), x["state"].to(DEV), scale=0.125,
                                  return_state=True)
        with np.errstate(invalid="ignore"):
            want, wS = ref.decay_attention(*(f64(x[name]) for name in "qkv"), f64(ld), f64(x["state"]), None, 0.125)
        assert np.array_equal(np.isfinite(f64(o)), np.isfinite(want)) and np.array_equal(np.isfinite(f64(S)), np.isfinite(wS))


def test_tensors_that_require_a_gradient_are_refused():
    # there is no backward pass, and a result without a graph would hide that
    def made(*shape, dtype=torch.float16):
        return torch.randn(shape, device=DEV).to(dtype)

    lin = [made(4, 64), made(32, 64), made(32), made(4, 32)]
    rope = [made(4, 2, 32), made(4, 1, 32), made(32), made(32), torch.zeros((4, 1), dtype=torch.int32, device=DEV),
            tk.rope_frequencies((16,), device=DEV)]
    decay = [made(1, 4, 2, 32), made(1, 4, 2, 32), made(1, 4, 2, 16), -torch.ones(2, device=DEV),
             made(1, 2, 32, 16, dtype=torch.float32)]
    for call, args in ((lambda *a: tk.linear(*a), lin), (lambda *a: tk.qk_norm_rope(*a, (16,)), rope),
                       (lambda *a: tk.decay_attention(*a, return_state=True), decay)):
        call(*args)
        for i, t in enumerate(args):
            if t.is_floating_point():
                t.requires_grad_()
                with pytest.raises(ValueError, match="no backward pass"):
                    call(*args)
                with torch.no_grad():
                    call(*args)
                t.requires_grad_(False)


def test_outputs_over_inputs_are_refused_and_parts_of_one_buffer_are_not():
    g = gen(5)
    x, w = rnd(g, (700, 512), "fp16").to(DEV), rnd(g, (512, 512), "fp16", 0.05).to(DEV)
    before = x.clone()
    for bad in (lambda: tk.linear(x, w, out=x), lambda: tk.linear(x[:512], w, out=w), lambda: tk.linear(x[1:], w, out=x[:-1]),
                lambda: tk.linear(x[:-1], w, residual=x[1:], out=x[:-1])):
        with pytest.raises(nc.NcodecError) as e:
            bad()
        assert e.value.status == nc.NCODEC_EINVAL
    assert torch.equal(x, before)
    buf = torch.zeros((700, 1024), dtype=torch.float16, device=DEV)
    buf[:, :512] = x
    tk.linear(buf[:, :512], w, out=buf[:, 512:])
    assert torch.equal(buf[:, :512], x) and torch.equal(buf[:, 512:], tk.linear(x, w))
    # heads of one buffer: q, k, v, the rotated q and k, and the attention's output
    T, H, D = 90, 2, 64
    buf = rnd(g, (2, T, 6 * H, D), "fp16").to(DEV)
    q, k, v, q2, k2, o = (buf[:, :, H * i:H * i + H] for i in range(6))
    pos, fr = tk.grid_positions(2, 9, 10, device=DEV), tk.rope_frequencies((16, 8, 8), device=DEV)
    ld = torch.tensor([-0.1, -0.02], device=DEV)
    apart = [t.contiguous() for t in (q, k, v)]
    a, b = tk.qk_norm_rope(apart[0].view(-1, H, D), apart[1].view(-1, H, D), None, None, pos, fr, (16, 8, 8))
    flat = [t.reshape(2 * T, H, D) if t.is_contiguous() else buf.view(2 * T, 6 * H, D)[:, H * i:H * i + H]
            for i, t in enumerate((q, k, v, q2, k2, o))]
    tk.qk_norm_rope(flat[0], flat[1], None, None, pos, fr, (16, 8, 8), q_out=flat[3], k_out=flat[4])
    assert torch.equal(flat[3], a) and torch.equal(flat[4], b)
    want = tk.decay_attention(a.view(2, T, H, D), b.view(2, T, H, D), apart[2], ld)
    tk.decay_attention(q2, k2, v, ld, out=o)
    assert torch.equal(o, want) and torch.equal(v, apart[2])
    for bad in (lambda: tk.qk_norm_rope(flat[0], flat[1], q_out=flat[1], k_out=flat[4]),
                lambda: tk.qk_norm_rope(flat[0], flat[1], q_out=flat[3], k_out=flat[3]),
                lambda: tk.decay_attention(q, k, v, ld, out=v), lambda: tk.decay_attention(q, k, v, ld, out=q)):
        with pytest.raises(nc.NcodecError) as e:
            bad()
        assert e.value.status == nc.NCODEC_EINVAL


@pytest.mark.parametrize("T", [0, 1, 80])
def test_no_tokens_leave_the_state_before_or_zeros_and_no_sequences_leave_nothing(T):
    # the states are written whether no token is there, or none is counted
    x = torch.ones((2, T, 1, 32), dtype=torch.float16, device=DEV)
    ld = torch.zeros(1, device=DEV)
    none = torch.zeros(2, dtype=torch.int32, device=DEV)
    S0 = torch.randn((2, 1, 32, 32), device=DEV)
    out = torch.full_like(S0, 7.0)
    tk.decay_attention(x, x, x, ld, S0, none, state_out=out)
    assert torch.equal(out, S0)
    tk.decay_attention(x, x, x, ld, None, none, state_out=out)
    assert bool((out == 0).all())
    o = tk.decay_attention(x[:0], x[:0], x[:0], ld, S0[:0], state_out=out[:0])
    assert o.shape == (0, T, 1, 32) and bool((out == 0).all())
