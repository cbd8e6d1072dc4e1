"""Token operators on torch tensors, and the mixer that they make.

``linear``, ``qk_norm_rope`` and ``decay_attention`` check their arguments, allocate outputs and workspace with
torch and call the library's entry points of the same names on the current stream of the tensors' device; every
value is computed in the HIP kernels.  They take float16 or bfloat16 tensors and strided views (the last dimension
contiguous) and raise :class:`ValueError` for tensors that do not fit together, :class:`NcodecError` for what the
library refuses, outputs that overlap an input or each other among it (parts of one buffer may be given, and what a
function says may be the same).  They have no backward pass: a tensor that requires a gradient is refused where torch records
gradients, and taken under ``torch.no_grad()``.  :class:`TokenMixer` runs them together: a layer
that reads the latents of all earlier frames through a state of fixed size.
"""
from __future__ import annotations

import ctypes

import torch

from . import ncodec as _nc
from .ncodec import ACTS, NCODEC_DTYPE_BF16, NCODEC_DTYPE_FP16

_DTYPES = {torch.float16: NCODEC_DTYPE_FP16, torch.bfloat16: NCODEC_DTYPE_BF16}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


_NO_BACKWARD = "no backward pass: call under torch.no_grad(), or with tensors that require no gradient"


def _dtype(x):
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError(_NO_BACKWARD)
    dt = _DTYPES.get(x.dtype)
    if dt is None or not x.is_cuda:
        raise ValueError(f"tensors must be float16 or bfloat16 on the GPU, not {x.dtype} on {x.device}")
    return dt


def _like(t, dtype, device, shape, what):
    """t has this type, device (index) and shape, its last dimension contiguous, and asks for no gradient."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(_NO_BACKWARD)
    if t.dtype != dtype or t.get_device() != device:
        raise ValueError(f"{what}: {t.dtype} on {t.device}, expected {dtype} on cuda:{device}")
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _raw_stream(index):
    return torch.cuda.current_stream(index).cuda_stream


# the same without building a Stream object, where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


def _call(fn, index, *args):
    """fn(*args, stream) on the current stream of device `index`."""
    if torch.cuda.current_device() == index:
        st = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _raw_stream(index))
    if st:
        _nc._check(st)


def linear(x, weight, bias=None, residual=None, act="none", gated=False, out=None):
    """``act(x W^T + b) + residual``; gated, with W = [W1; W2]: ``act(x W1^T + b1) * (x W2^T + b2) + residual``.

    x: (..., k) whose rows are evenly spaced, weight: (n, k), gated (2n, k), bias: (n) or (2n), residual: (..., n).
    act: "none", "lrelu" (slope 0.1), "wsilu" (v sigmoid(4v)), "silu" or "gelu".  ``out`` may be ``residual``.
    Sums and the epilogue are float32, rounded once."""
    dt = _dtype(x)
    act_code = ACTS.get(act)
    if act_code is None:
        raise ValueError(f"act must be one of {sorted(ACTS)}")
    xs, ws = x.shape, weight.shape
    _need(len(xs) >= 1 and len(ws) == 2, "x needs a dimension, weight two")
    k, rows = xs[-1], ws[0]
    _need(not gated or rows % 2 == 0, "a gated weight has an even number of rows")
    n = rows // 2 if gated else rows
    dtype, device = x.dtype, x.get_device()
    if x.stride(-1) != 1 and k > 1:
        raise ValueError("x: the last dimension must be contiguous")
    _like(weight, dtype, device, (rows, k), "weight")
    if bias is not None:
        _like(bias, dtype, device, (rows,), "bias")
    ys = (*xs[:-1], n)
    if out is None:
        y = x.new_empty(ys)
    else:
        y = out
        _like(y, dtype, device, ys, "out")
    flat = len(xs) == 2
    x2, y2 = (x, y) if flat else (_flat(x, "x"), _flat(y, "out"))
    ldr = 0
    if residual is not None:
        _like(residual, dtype, device, ys, "residual")
        ldr = (residual if flat else _flat(residual, "residual")).stride(0)
    m = x2.shape[0]
    if m == 1:  # the stride of a dimension with one entry means nothing
        ldx, ldy, ldr = k, n, n
    else:
        ldx, ldy = x2.stride(0), y2.stride(0)
    shape = _nc.ncodec_linear_shape(dt, act_code, 1 if gated else 0, 0, m, n, k, ldx,
                                    weight.stride(0) if rows > 1 else k, ldr, ldy)
    _call(_nc.load_library().ncodec_linear, device, ctypes.byref(shape), x.data_ptr(), weight.data_ptr(), _ptr(bias),
          _ptr(residual), y.data_ptr())
    return y


def _flat(t, what):
    """t with its leading dimensions as one, without a copy."""
    try:
        return t.view(-1, t.shape[-1]) if t.shape[-1] and t.numel() else t.reshape(-1, t.shape[-1])
    except RuntimeError:
        raise ValueError(f"{what}: its rows must be evenly spaced") from None


def rope_frequencies(sections, base=10000.0, device="cuda:0"):
    """Radians per step of each pair, float32: pair i of an axis with p pairs turns by base^(-i / p) a step."""
    return torch.cat([base ** (-torch.arange(p, dtype=torch.float64) / max(p, 1)) for p in sections]).to(
        dtype=torch.float32, device=device)


def grid_positions(frames, height, width, t0=0, device="cuda:0"):
    """(frames * height * width, 3) int32 positions (t, h, w) of whole frames in raster order, the first at t0."""
    t, h, w = (torch.arange(n, dtype=torch.int32, device=device) for n in (frames, height, width))
    return torch.stack(torch.meshgrid(t + t0, h, w, indexing="ij"), -1).reshape(-1, 3).contiguous()


def qk_norm_rope(q, k, q_weight=None, k_weight=None, positions=None, freq=None, sections=(), eps=1e-6, norm=True,
                 interleaved=False, q_out=None, k_out=None):
    """RMS norm of every head of q and k and the rotation by each token's position; returns (q', k').

    q: (tokens, q_heads, dim), k: (tokens, k_heads, dim), weights: (dim) or None (ones); norm=False rotates only.
    positions: (tokens, axes) int32 with axes up to 3, sections: pairs given to each axis, freq: (sum of sections)
    float32 radians per step (:func:`rope_frequencies`).  Without sections there is no rotation.  ``q_out`` and
    ``k_out`` may be q and k themselves."""
    dt = _dtype(q)
    qs, ks = q.shape, k.shape
    _need(len(qs) == 3 and len(ks) == 3, "q and k must be (tokens, heads, dim)")
    T, hq, D = qs
    hk = ks[1]
    dtype, device = q.dtype, q.get_device()
    _like(q, dtype, device, qs, "q")
    _like(k, dtype, device, (T, hk, D), "k")
    _need(norm or (q_weight is None and k_weight is None), "weights without a norm")
    if q_weight is not None:
        _like(q_weight, dtype, device, (D,), "q_weight")
    if k_weight is not None:
        _like(k_weight, dtype, device, (D,), "k_weight")
    axes = len(sections)
    pos = fr = None
    if axes:
        _need(axes <= 3, "at most three axes")
        _need(positions is not None and freq is not None, "a rotation needs positions and freq")
        _like(positions, torch.int32, device, (T, axes), "positions")
        _need(positions.is_contiguous(), "positions must be contiguous")
        _like(freq, torch.float32, device, (sum(sections),), "freq")
        pos, fr = positions.data_ptr(), freq.data_ptr()
    if q_out is None:
        q_out = q.new_empty((T, hq, D))
    else:
        _like(q_out, dtype, device, qs, "q_out")
    if k_out is None:
        k_out = q.new_empty((T, hk, D))
    else:
        _like(k_out, dtype, device, ks, "k_out")
    a, b, c, d = q.stride(), k.stride(), q_out.stride(), k_out.stride()
    shape = _nc.ncodec_qk_shape(dt, 1 if norm else 0, axes, (*sections, 0, 0, 0)[:3], 1 if interleaved else 0, hq, hk, D,
                                eps, 0, T, a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1])
    _call(_nc.load_library().ncodec_qk_norm_rope, device, ctypes.byref(shape), q.data_ptr(), k.data_ptr(),
          _ptr(q_weight), _ptr(k_weight), pos, fr, q_out.data_ptr(), k_out.data_ptr())
    return q_out, k_out


def decay_attention(q, k, v, log_decay, state=None, lengths=None, scale=None, return_state=False, out=None,
                    state_out=None):
    """Linear attention with a decay for each head: S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t S_t.

    q: (batch, tokens, heads, dim), k: (batch, tokens, kv_heads, dim), v: (batch, tokens, kv_heads, value_dim),
    log_decay: (heads) float32 <= 0, state: (batch, heads, dim, value_dim) float32 before the first token (None:
    zero), lengths: (batch) int32 tokens of each sequence (None: all; past them outputs are zero), scale: default
    dim^-0.5.  Returns o (batch, tokens, heads, value_dim), with return_state (o, state after the last token).
    ``state_out`` may be ``state`` itself: one token per call is the recurrent form.  Sequences without tokens leave
    their state as it was (None: zeros)."""
    dt = _dtype(q)
    qs, ks, vs = q.shape, k.shape, v.shape
    _need(len(qs) == 4 and len(ks) == 4 and len(vs) == 4, "q, k and v must be (batch, tokens, heads, dim)")
    B, T, H, D = qs
    hk, V = ks[2], vs[3]
    _need(D >= 1, "q needs a head dimension")
    dtype, device = q.dtype, q.get_device()
    _like(q, dtype, device, qs, "q")
    _like(k, dtype, device, (B, T, hk, D), "k")
    _like(v, dtype, device, (B, T, hk, V), "v")
    _like(log_decay, torch.float32, device, (H,), "log_decay")
    if lengths is not None:
        _like(lengths, torch.int32, device, (B,), "lengths")
    if state is not None:
        _like(state, torch.float32, device, (B, H, D, V), "state")
        _need(state.is_contiguous(), "state must be contiguous")
    if state_out is not None:
        _like(state_out, torch.float32, device, (B, H, D, V), "state_out")
        _need(state_out.is_contiguous(), "state_out must be contiguous")
    elif return_state:
        state_out = q.new_empty((B, H, D, V), dtype=torch.float32)
    if out is None:
        out = q.new_empty((B, T, H, V))
    else:
        _like(out, dtype, device, (B, T, H, V), "out")
    shape = _nc.ncodec_decay_shape(dt, H, hk, D, V, D ** -0.5 if scale is None else scale, B, T, *q.stride()[:3],
                                   *k.stride()[:3], *v.stride()[:3], *out.stride()[:3])
    lib = _nc.load_library()
    ref = ctypes.byref(shape)
    need = lib.ncodec_decay_attention_workspace_bytes(ref)
    ws = q.new_empty(need, dtype=torch.uint8) if need else None
    _call(lib.ncodec_decay_attention, device, ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(),
          _ptr(lengths), _ptr(state), _ptr(state_out), out.data_ptr(), _ptr(ws), need)
    return (out, state_out) if return_state else out
