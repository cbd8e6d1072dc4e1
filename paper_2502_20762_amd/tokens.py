"""Token operators on torch tensors, and the mixer that they make.

``linear``, ``qk_norm_rope`` and ``decay_attention`` check their arguments, allocate outputs and workspace with
torch and call the library's entry points of the same names on the current stream of the tensors' device; every
value is computed in the HIP kernels.  They take float16 or bfloat16 tensors and strided views (the last dimension
contiguous) and raise :class:`ValueError` for tensors that do not fit together, :class:`NcodecError` for what the
library refuses.  :class:`TokenMixer` runs them together: the layer of a temporal prior that reads the latents of
all earlier frames through a state of fixed size.
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


def _dtype(x):
    dt = _DTYPES.get(x.dtype)
    if dt is None or not x.is_cuda:
        raise ValueError(f"tensors must be float16 or bfloat16 on the GPU, not {x.dtype} on {x.device}")
    return dt


def _like(t, x, what, shape=None, dtype=None):
    """t sits with x: device, type and (if given) shape, its last dimension contiguous."""
    if t.dtype != (dtype or x.dtype) or t.get_device() != x.get_device():
        raise ValueError(f"{what}: {t.dtype} on {t.device}, expected {dtype or x.dtype} on {x.device}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
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


def _row_stride(t, i, width):
    """Stride of dimension i, or the packed one where the dimension has one entry (its stride means nothing)."""
    return t.stride(i) if t.shape[i] > 1 else max(t.stride(i), width)


def linear(x, weight, bias=None, residual=None, act="none", gated=False, out=None):
    """``act(x W^T + b) + residual``; gated, with W = [W1; W2]: ``act(x W1^T + b1) * (x W2^T + b2) + residual``.

    x: (..., k) whose rows are evenly spaced, weight: (n, k), gated (2n, k), bias: (n) or (2n), residual: (..., n).
    act: "none", "lrelu" (slope 0.1), "wsilu" (v sigmoid(4v)), "silu" or "gelu".  ``out`` may be ``residual``.
    Sums and the epilogue are float32, rounded once."""
    dt = _dtype(x)
    if act not in ACTS:
        raise ValueError(f"act must be one of {sorted(ACTS)}")
    _need(x.dim() >= 1 and weight.dim() == 2, "x needs a dimension, weight two")
    k, rows = x.shape[-1], weight.shape[0]
    _need(not gated or rows % 2 == 0, "a gated weight has an even number of rows")
    n = rows // 2 if gated else rows
    _like(x, x, "x")
    _like(weight, x, "weight", (rows, k))
    lead = x.shape[:-1]
    x2 = x if x.dim() == 2 else _flat(x, "x")
    if bias is not None:
        _like(bias, x, "bias", (rows,))
    if residual is not None:
        _like(residual, x, "residual", lead + (n,))
    y = out
    if y is None:
        y = x.new_empty(lead + (n,))
    else:
        _like(y, x, "out", lead + (n,))
    y2 = y if y.dim() == 2 else _flat(y, "out")
    r2 = None if residual is None else residual if residual.dim() == 2 else _flat(residual, "residual")
    shape = _nc.ncodec_linear_shape(dt, ACTS[act], 1 if gated else 0, 0, x2.shape[0], n, k, _row_stride(x2, 0, k),
                                    _row_stride(weight, 0, k), 0 if r2 is None else _row_stride(r2, 0, n),
                                    _row_stride(y2, 0, n))
    _call(_nc.load_library().ncodec_linear, x.get_device(), ctypes.byref(shape), _ptr(x), _ptr(weight), _ptr(bias),
          _ptr(residual), _ptr(y))
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
    _need(q.dim() == 3 and k.dim() == 3, "q and k must be (tokens, heads, dim)")
    T, hq, D = q.shape
    hk = k.shape[1]
    _like(q, q, "q")
    _like(k, q, "k", (T, hk, D))
    for w in (q_weight, k_weight):
        if w is not None:
            _need(norm, "weights without a norm")
            _like(w, q, "norm weight", (D,))
    axes = len(sections)
    _need(axes <= 3, "at most three axes")
    if axes:
        _need(positions is not None and freq is not None, "a rotation needs positions and freq")
        _like(positions, q, "positions", (T, axes), torch.int32)
        _need(positions.is_contiguous(), "positions must be contiguous")
        _like(freq, q, "freq", (sum(sections),), torch.float32)
    if q_out is None:
        q_out = q.new_empty((T, hq, D))
    else:
        _like(q_out, q, "q_out", (T, hq, D))
    if k_out is None:
        k_out = q.new_empty((T, hk, D))
    else:
        _like(k_out, q, "k_out", (T, hk, D))
    shape = _nc.ncodec_qk_shape(dt, 1 if norm else 0, axes, tuple(sections) + (0,) * (3 - axes),
                                1 if interleaved else 0, hq, hk, D, eps, 0, T, q.stride(0), q.stride(1), k.stride(0),
                                k.stride(1), q_out.stride(0), q_out.stride(1), k_out.stride(0), k_out.stride(1))
    _call(_nc.load_library().ncodec_qk_norm_rope, q.get_device(), ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(q_weight),
          _ptr(k_weight), _ptr(positions) if axes else None, _ptr(freq) if axes else None, _ptr(q_out), _ptr(k_out))
    return q_out, k_out


def decay_attention(q, k, v, log_decay, state=None, lengths=None, scale=None, return_state=False, out=None,
                    state_out=None):
    """Linear attention with a decay for each head: S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t S_t.

    q: (batch, tokens, heads, dim), k: (batch, tokens, kv_heads, dim), v: (batch, tokens, kv_heads, value_dim),
    log_decay: (heads) float32 <= 0, state: (batch, heads, dim, value_dim) float32 before the first token (None:
    zero), lengths: (batch) int32 tokens of each sequence (None: all; past them outputs are zero), scale: default
    dim^-0.5.  Returns o (batch, tokens, heads, value_dim), with return_state (o, state after the last token).
    ``state_out`` may be ``state`` itself: one token per call is the recurrent form."""
    dt = _dtype(q)
    _need(q.dim() == 4 and k.dim() == 4 and v.dim() == 4, "q, k and v must be (batch, tokens, heads, dim)")
    B, T, H, D = q.shape
    hk, V = k.shape[2], v.shape[3]
    _need(D >= 1, "q needs a head dimension")
    _like(q, q, "q")
    _like(k, q, "k", (B, T, hk, D))
    _like(v, q, "v", (B, T, hk, V))
    _like(log_decay, q, "log_decay", (H,), torch.float32)
    if lengths is not None:
        _like(lengths, q, "lengths", (B,), torch.int32)
    if state is not None:
        _like(state, q, "state", (B, H, D, V), torch.float32)
        _need(state.is_contiguous(), "state must be contiguous")
    if state_out is None:
        if return_state:
            state_out = q.new_empty((B, H, D, V), dtype=torch.float32)
    else:
        _like(state_out, q, "state_out", (B, H, D, V), torch.float32)
        _need(state_out.is_contiguous(), "state_out must be contiguous")
    if out is None:
        out = q.new_empty((B, T, H, V))
    else:
        _like(out, q, "out", (B, T, H, V))
    shape = _nc.ncodec_decay_shape(dt, H, hk, D, V, D ** -0.5 if scale is None else scale, B, T, *q.stride()[:3],
                                   *k.stride()[:3], *v.stride()[:3], *out.stride()[:3])
    lib = _nc.load_library()
    ref = ctypes.byref(shape)
    need = lib.ncodec_decay_attention_workspace_bytes(ref)
    ws = q.new_empty(need, dtype=torch.uint8) if need else None
    _call(lib.ncodec_decay_attention, q.get_device(), ref, _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(lengths),
          _ptr(state), _ptr(state_out), _ptr(out), _ptr(ws), need)
    return (out, state_out) if return_state else out
