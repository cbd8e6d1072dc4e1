"""Mixers over latent tokens: layers that see more than the frame before.

The codec's own memory of the past is one frame: the context f_{t-1} and the latent yhat_{t-1} that its prior reads.
:class:`TokenMixer` reads the decoded latents of a stream as tokens, one per position (t, h, w) of the 1/16 grid, and
keeps all of them in a state of fixed size (heads x head_dim x head_dim float32), so that a frame costs the same
however long the stream is.  :class:`CacheMixer` is the same layer with softmax attention over a window of tokens and
the first ones, or over the heaviest ones of a budget: an encoder has all tokens of a clip and runs them as a prompt, a
decoder has them one after the other and keeps their keys and values in the pages of a :class:`TokenCache`.  Encoder
and decoder both hold yhat after every frame, so both can run them.  They stand beside the codec: what they return is
for the caller, and the codec's own prior, entropy model and bitstream do not read it.

``python -m paper_2502_20762_amd.mixer`` codes a short synthetic sequence with random-init weights and runs both mixers
beside the encoder.
"""
from __future__ import annotations

import math

import torch

from .tokens import (cache_append, cache_evict, decay_attention, grid_positions, linear, paged_attention, qk_norm_rope,
                     rope_frequencies, window_attention)


class TokenMixer:
    """x + Wo attention(norm and rotation of Wqkv x), then x + W2 (wsilu(W1a x) * (W1b x)), with random-init weights.

    channels: C of the codec; heads query heads of head_dim over kv_heads key and value heads; expand: width of the
    gated layer over C.  Head h keeps a token for about 2^(4 + 8 h / heads) tokens.  ``weights`` (see
    :meth:`parameters`) replace the random ones."""

    def __init__(self, channels, heads=4, kv_heads=None, head_dim=64, expand=2, dtype=torch.float16, device="cuda:0",
                 seed=0, weights=None):
        self.C, self.H, self.K, self.D = channels, heads, kv_heads or heads, head_dim
        self.F, self.dtype, self.device = expand * channels, dtype, torch.device(device)
        shapes = self.parameters()
        if weights is None:
            g = torch.Generator()
            g.manual_seed(seed)
            weights = {}
            for name, shape in shapes.items():
                if len(shape) == 2:  # the projections back to x are small, so that a layer stays near the identity
                    w = torch.randn(shape, generator=g) * ((0.25 if name in ("wo", "w2") else 1.0) / math.sqrt(shape[1]))
                else:
                    w = torch.ones(shape) if name in ("q_norm", "k_norm") else torch.zeros(shape)
                weights[name] = w
        self.w = {}
        for name, shape in shapes.items():
            if tuple(weights[name].shape) != shape:
                raise ValueError(f"{name}: shape {tuple(weights[name].shape)}, expected {shape}")
            self.w[name] = weights[name].to(device=self.device, dtype=dtype).contiguous()
        part = head_dim // 2 // 3
        self.sections = (head_dim // 2 - 2 * part, part, part)  # pairs for t, h, w
        self.freq = rope_frequencies(self.sections, device=self.device)
        keep = 2.0 ** -(4 + 8 * torch.arange(heads, dtype=torch.float64) / heads)
        self.log_decay = torch.log1p(-keep).to(dtype=torch.float32, device=self.device)

    def parameters(self):
        """Name and shape of every weight."""
        C, H, K, D, F = self.C, self.H, self.K, self.D, self.F
        return {"wqkv": ((H + 2 * K) * D, C), "q_norm": (D,), "k_norm": (D,), "wo": (C, H * D), "bo": (C,),
                "w1": (2 * F, C), "b1": (2 * F,), "w2": (C, F), "b2": (C,)}

    def new_state(self, batch=1):
        """The state of streams that have seen nothing."""
        return torch.zeros((batch, self.H, self.D, self.D), device=self.device)

    def __call__(self, x, positions, state, lengths=None):
        """x: (batch, tokens, C); positions: (tokens, 3) int32, the same for every stream of the batch; state: moved on
        in place past the tokens; lengths: (batch) int32 tokens of each stream (None: all).  Returns (batch, tokens, C)."""
        q, k, v = self._project(x, positions)
        o, _ = decay_attention(q, k, v, self.log_decay, state, lengths, return_state=True, state_out=state)
        return self._finish(x, o)

    def _project(self, x, positions):
        """Queries, keys and values of x (batch, tokens, C), normed and rotated, (batch, tokens, heads, dim) each."""
        B, T, C = x.shape
        H, K, D, w = self.H, self.K, self.D, self.w
        qkv = linear(x, w["wqkv"]).view(B * T, H + 2 * K, D)
        q, k = qkv[:, :H], qkv[:, H:H + K]
        if B > 1:
            positions = positions.repeat(B, 1)
        qk_norm_rope(q, k, w["q_norm"], w["k_norm"], positions, self.freq, self.sections, q_out=q, k_out=k)
        qkv = qkv.view(B, T, H + 2 * K, D)
        return qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:]

    def _finish(self, x, o):
        """What follows the attention's output o, (batch, tokens, heads, dim)."""
        B, T, C = x.shape
        w = self.w
        x = linear(o.view(B, T, self.H * self.D), w["wo"], w["bo"], residual=x)
        h = linear(x, w["w1"], w["b1"], act="wsilu", gated=True)
        return linear(h, w["w2"], w["b2"], residual=x)

    def frame(self, yhat, t, state):
        """The mixer over the latent of frame t, (C, h, w) as ``Codec.get_state`` returns it; returns the same shape."""
        C, h, w = yhat.shape
        x = yhat.reshape(C, h * w).t().contiguous().to(self.dtype)
        y = self(x[None], grid_positions(1, h, w, t0=t, device=self.device), state)
        return y[0].t().reshape(C, h, w)


class TokenCache:
    """Keys and values of the latest tokens of a batch of streams, in pages.

    capacity: tokens of a stream at most.  With ``keep`` a cache that would overflow is cut back first, to the first
    ``sinks`` and the latest ``recent`` tokens and, up to ``keep`` tokens in all, the heaviest of the others by the
    attention weights that :meth:`attend` and :meth:`weigh_prompt` have given them (``weigh=False``: none are summed, for a
    ``keep`` that the first and the latest fill); ``keep`` has to leave room for the tokens that come at once.  Without ``keep`` an append that
    does not fit is refused."""

    def __init__(self, batch, capacity, kv_heads, head_dim, value_dim=None, page_size=16, keep=None, sinks=0, recent=0,
                 weigh=True, dtype=torch.float16, device="cuda:0"):
        columns = -(-capacity // page_size)
        if keep is not None and not 0 < keep < capacity:
            raise ValueError("keep must be in [1, capacity)")
        if keep is not None and (sinks < 0 or recent < 0 or sinks + recent > keep):
            raise ValueError("sinks + recent must be in [0, keep]")
        self.capacity, self.keep, self.sinks, self.recent, self.weigh = capacity, keep, sinks, recent, weigh
        self.most = 0  # tokens of the fullest stream, at most: known without asking the GPU,
        self.exact = True  # and just that many as long as all streams get the same
        pages = batch * columns
        count = 2 * pages if keep is not None else pages  # an eviction copies to pages that are free
        self.k = torch.zeros((count, page_size, kv_heads, head_dim), dtype=dtype, device=device)
        self.v = torch.zeros((count, page_size, kv_heads, value_dim or head_dim), dtype=dtype, device=device)
        tables = torch.arange(count, dtype=torch.int32, device=device).view(-1, batch, columns)
        self.table, self.free = tables[0], tables[1] if keep is not None else None
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=device)
        self.mass = torch.zeros((batch, kv_heads, columns * page_size), device=device) if keep is not None else None

    def append(self, k, v, counts=None):
        """Adds tokens, k and v (batch, tokens, kv_heads, dim); counts: (batch) int32 of each stream (None: all).  The
        host waits for the GPU only where streams of different length come near the capacity."""
        T = k.shape[1]
        new = T if counts is None else counts.clamp(0, T)
        exact = self.exact and counts is None
        most = self.most + T
        if most > self.capacity and not exact and len(self.lengths):
            most, exact = int((self.lengths + new).max()), True
        if most > self.capacity:
            left = most  # of the fullest stream, once it is cut back
            if self.keep is not None:
                left = min(self.most, self.keep) + T if counts is None else int((self.lengths.clamp(max=self.keep) + new).max())
            if left > self.capacity:  # before anything is let go
                raise ValueError(f"{T} tokens do not fit: a stream would hold {left}, and the cache has room for {self.capacity}")
            # of none of these tokens: whatever the write refuses, it does so here
            none = torch.zeros_like(self.lengths if counts is None else counts)
            cache_append(k, v, self.k, self.v, self.table, self.lengths, none, self.mass)
            self.evict()
            most = left
        cache_append(k, v, self.k, self.v, self.table, self.lengths, counts, self.mass)
        self.lengths += new
        self.most, self.exact = most, exact

    def attend(self, q, window=None, sinks=0):
        """Attention of each stream's last token, q (batch, heads, dim)."""
        return paged_attention(q, self.k, self.v, self.table, self.lengths, window, sinks,
                               mass=self.mass if self.weigh else None)

    def weigh_prompt(self, q, counts=None, window=None, sinks=0):
        """Adds the weights that the first tokens of all streams, q (batch, tokens, heads, dim), give to those up to
        themselves, as :meth:`attend` would have after each of them; counts: as in :meth:`append`.  Some queries of every
        stream at once, as many as fill a GPU, each a sequence of its own over the same pages."""
        if not self.weigh or self.mass is None:
            return
        B, T, H, D = q.shape
        n = max(1, 64 // max(B, 1))
        for i in range(0, T, n):
            part = q[:, i:i + n]
            seen = torch.arange(i + 1, i + 1 + part.shape[1], dtype=torch.int32, device=q.device).repeat(B, 1)
            if counts is not None:
                seen = seen * (seen <= counts[:, None])
            mass = torch.zeros((B, part.shape[1], *self.mass.shape[1:]), device=q.device)
            paged_attention(part.reshape(-1, H, D), self.k, self.v, self.table.repeat_interleave(part.shape[1], 0),
                            seen.reshape(-1), window, sinks, mass=mass.flatten(0, 1))
            self.mass += mass.sum(1)

    def evict(self):
        """Cuts every stream back to ``keep`` tokens; returns their old positions."""
        if self.keep is None:
            raise ValueError("a cache without keep lets go of nothing")
        self.lengths, self.mass, kept = cache_evict(self.k, self.v, self.table, self.lengths, self.mass, self.keep,
                                                    self.free, self.sinks, self.recent)
        self.table, self.free = self.free, self.table
        self.most = min(self.most, self.keep)
        return kept


class CacheMixer(TokenMixer):
    """The layer of :class:`TokenMixer` with softmax attention: a token sees the latest ``window`` tokens, itself among
    them (None: all), and the first ``sinks``."""

    def __init__(self, channels, heads=4, kv_heads=None, head_dim=64, expand=2, window=None, sinks=0, **more):
        super().__init__(channels, heads, kv_heads, head_dim, expand, **more)
        self.window, self.sinks = window, sinks

    def new_cache(self, capacity, batch=1, page_size=16, keep=None, recent=0):
        """A cache of streams that have seen nothing.  Without a window, ``keep`` and ``recent`` bound it as they do a
        :class:`TokenCache`.  With one, a cache with room for more than the window and the first tokens lets go of what no
        later token sees, and takes streams of any length, whose prompt has to fit it."""
        weigh = self.window is None
        if not weigh:
            if keep is not None:
                raise ValueError("a cache that keeps the heaviest tokens goes with window=None")
            recent = self.window - 1
            if max(1, self.sinks + recent) < capacity:
                keep = max(1, self.sinks + recent)
        return TokenCache(batch, capacity, self.K, self.D, None, page_size, keep, self.sinks, recent, weigh, self.dtype,
                          self.device)

    def __call__(self, x, positions, cache=None, lengths=None):
        """The prompt form: x (batch, tokens, C) are the first tokens of their streams, positions (tokens, 3) int32;
        lengths: (batch) int32 tokens of each stream (None: all).  ``cache``, empty before, holds them afterwards, one with
        a budget their weights too, which takes longer than the prompt itself (8,160 tokens of 4 heads of 64: 7.5 ms, one by
        one 241).  Returns (batch, tokens, C)."""
        q, k, v = self._project(x, positions)
        if cache is not None:
            if cache.most:
                raise ValueError("a prompt begins its streams: the cache must be empty")
            cache.append(k, v, lengths)
            cache.weigh_prompt(q, lengths, self.window, self.sinks)
        return self._finish(x, window_attention(q, k, v, self.window, self.sinks, lengths))

    def step(self, x, position, cache):
        """The next token of every stream, x (batch, C) at position (1, 3); returns (batch, C)."""
        x = x[:, None]
        q, k, v = self._project(x, position)
        cache.append(k, v)
        return self._finish(x, cache.attend(q[:, 0], self.window, self.sinks)[:, None])[:, 0]

    def frame(self, yhat, t, cache):
        """The mixer over the latent of frame t, (C, h, w), token by token; returns the same shape."""
        C, h, w = yhat.shape
        x = yhat.reshape(C, h * w).t().contiguous().to(self.dtype)
        positions = grid_positions(1, h, w, t0=t, device=self.device)
        y = [self.step(x[i:i + 1], positions[i:i + 1], cache) for i in range(h * w)]
        return torch.cat(y).t().reshape(C, h, w)


def main():
    import synth

    from .ncodec import Codec

    C, H, W = 64, 64, 64
    device = "cuda:0"
    codec = Codec(H, W, C, 2, 2, "fp16", synth.make_weights(C, 2, 2), device=device)
    mixer = TokenMixer(C, device=device)
    state = mixer.new_state()
    exact = CacheMixer(C, sinks=4, device=device)
    cache = exact.new_cache(24, keep=16, recent=4)
    for t, frame in enumerate(synth.frame_sequence("tiny")):
        codec.encode(torch.from_numpy(frame).to(device))
        _, yhat = codec.get_state()
        y = mixer.frame(yhat, t, state)
        z = exact.frame(yhat, t, cache)
        torch.cuda.synchronize()
        print(f"frame {t}: latent {tuple(yhat.shape)}, mixed rms {float(y.float().square().mean().sqrt()):.4f}, "
              f"state {state.numel() * 4} bytes, rms {float(state.square().mean().sqrt()):.4f}; over the cache "
              f"{float(z.float().square().mean().sqrt()):.4f}, {int(cache.lengths[0])} tokens held")


if __name__ == "__main__":
    main()
