"""A mixer over latent tokens: a layer that sees every earlier frame.

The codec's own memory of the past is one frame: the context f_{t-1} and the latent yhat_{t-1} that its prior reads.
:class:`TokenMixer` reads the decoded latents of a stream as tokens, one per position (t, h, w) of the 1/16 grid, and
keeps all of them in a state of fixed size (heads x head_dim x head_dim float32), so that a frame costs the same
however long the stream is.  Encoder and decoder both hold yhat after every frame, so both can run it.  It stands
beside the codec: what it returns is for the caller, and the codec's own prior, entropy model and bitstream do not
read it.

``python -m paper_2502_20762_amd.mixer`` codes a short synthetic sequence with random-init weights and runs the mixer
beside the encoder.
"""
from __future__ import annotations

import math

import torch

from .tokens import decay_attention, grid_positions, linear, qk_norm_rope, rope_frequencies


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
        B, T, C = x.shape
        H, K, D, w = self.H, self.K, self.D, self.w
        qkv = linear(x, w["wqkv"]).view(B * T, H + 2 * K, D)
        q, k = qkv[:, :H], qkv[:, H:H + K]
        if B > 1:
            positions = positions.repeat(B, 1)
        qk_norm_rope(q, k, w["q_norm"], w["k_norm"], positions, self.freq, self.sections, q_out=q, k_out=k)
        qkv = qkv.view(B, T, H + 2 * K, D)
        o, _ = decay_attention(qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:], self.log_decay, state, lengths,
                               return_state=True, state_out=state)
        x = linear(o.view(B, T, H * D), w["wo"], w["bo"], residual=x)
        h = linear(x, w["w1"], w["b1"], act="wsilu", gated=True)
        return linear(h, w["w2"], w["b2"], residual=x)

    def frame(self, yhat, t, state):
        """The mixer over the latent of frame t, (C, h, w) as ``Codec.get_state`` returns it; returns the same shape."""
        C, h, w = yhat.shape
        x = yhat.reshape(C, h * w).t().contiguous().to(self.dtype)
        y = self(x[None], grid_positions(1, h, w, t0=t, device=self.device), state)
        return y[0].t().reshape(C, h, w)


def main():
    import synth

    from .ncodec import Codec

    C, H, W = 64, 64, 64
    device = "cuda:0"
    codec = Codec(H, W, C, 2, 2, "fp16", synth.make_weights(C, 2, 2), device=device)
    mixer = TokenMixer(C, device=device)
    state = mixer.new_state()
    for t, frame in enumerate(synth.frame_sequence("tiny")):
        codec.encode(torch.from_numpy(frame).to(device))
        _, yhat = codec.get_state()
        y = mixer.frame(yhat, t, state)
        torch.cuda.synchronize()
        print(f"frame {t}: latent {tuple(yhat.shape)}, mixed rms {float(y.float().square().mean().sqrt()):.4f}, "
              f"state {state.numel() * 4} bytes, rms {float(state.square().mean().sqrt()):.4f}")


if __name__ == "__main__":
    main()
