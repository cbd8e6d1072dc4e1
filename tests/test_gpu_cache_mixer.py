"""The softmax attentions and their cache together: the mixer over a cache against the float64 oracle, and its ways of
taking a stream.

Each of the seven rounded intermediates contributes about one unit roundoff of relative error, the layers' gain is
below two: 16 u of relative rms holds the sum with room for their worst alignment."""
import numpy as np
import pytest
import torch

import synth
from attention_util import DEV, f64
from oracle import tokens as ref
from paper_2502_20762_amd.mixer import CacheMixer, TokenCache, main
from paper_2502_20762_amd.ncodec import Codec
from paper_2502_20762_amd.tokens import grid_positions
from test_gpu_mixer import U, rms

pytestmark = pytest.mark.gpu


def oracle_mixer(m, x, pos, lengths=None):
    w = {k: f64(v) for k, v in m.w.items()}
    B, T, C = x.shape
    H, K, D = m.H, m.K, m.D
    qkv = ref.linear(x.reshape(B * T, C), w["wqkv"]).reshape(B * T, H + 2 * K, D)
    pos = np.tile(pos, (B, 1))
    q = ref.norm_rope(qkv[:, :H], w["q_norm"], pos, f64(m.freq), m.sections)
    k = ref.norm_rope(qkv[:, H:H + K], w["k_norm"], pos, f64(m.freq), m.sections)
    o = ref.window_attention(q.reshape(B, T, H, D), k.reshape(B, T, K, D), qkv[:, H + K:].reshape(B, T, K, D), m.window,
                             m.sinks, lengths, D ** -0.5)
    x = x.reshape(B * T, C)
    y = ref.linear(o.reshape(B * T, H * D), w["wo"], w["bo"], x)
    h = ref.linear(y, w["w1"], w["b1"], None, "wsilu", True)
    return ref.linear(h, w["w2"], w["b2"], y).reshape(B, T, C)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("C,heads,kv,dim,window,sinks", [(64, 4, 4, 64, None, 0), (128, 4, 2, 32, 40, 5), (256, 2, 1, 128, 17, 1)])
def test_prompt_and_steps_against_the_oracle(C, heads, kv, dim, window, sinks, dtype):
    m = CacheMixer(C, heads, kv, dim, window=window, sinks=sinks, dtype=dtype, device=DEV)
    g = torch.Generator()
    g.manual_seed(3)
    x = torch.randn((2, 90, C), generator=g).to(dtype).to(DEV)
    pos = grid_positions(2, 5, 9, t0=7, device=DEV)
    want = oracle_mixer(m, f64(x), f64(pos))
    assert rms(m(x, pos), want) <= 16 * U[dtype]
    # a prompt of 60, then token by token
    cache = m.new_cache(90, batch=2)
    head = m(x[:, :60].contiguous(), pos[:60], cache)
    tail = torch.stack([m.step(x[:, i], pos[i:i + 1], cache) for i in range(60, 90)], 1)
    torch.cuda.synchronize()
    assert rms(torch.cat([head, tail], 1), want) <= 16 * U[dtype]
    assert cache.lengths.tolist() == [90, 90] and cache.most == 90


def test_streams_of_different_length():
    m = CacheMixer(64, window=30, sinks=2, device=DEV)
    x = torch.randn((3, 41, 64), device=DEV).half()
    pos = grid_positions(1, 1, 41, device=DEV)
    lengths = torch.tensor([40, 0, 17], dtype=torch.int32, device=DEV)
    cache = m.new_cache(41, batch=3)
    m(x[:, :40].contiguous(), pos[:40], cache, lengths)
    assert cache.lengths.tolist() == [40, 0, 17] and cache.most == 40
    last = x.gather(1, lengths.long()[:, None, None].expand(3, 1, 64))[:, 0]
    y = m.step(last, pos[40:], cache)
    for b, n in enumerate([40, 0, 17]):
        alone = m.new_cache(41)
        if n:
            m(x[b:b + 1, :n].contiguous(), pos[:n], alone)
        assert rms(y[b:b + 1], f64(m.step(last[b:b + 1], pos[40:], alone))) <= 16 * U[torch.float16]


@pytest.mark.parametrize("window,sinks,capacity", [(30, 3, 40), (30, 0, 30), (2, 1, 5), (17, 20, 64), (1, 0, 4)])
def test_a_window_takes_streams_of_any_length(window, sinks, capacity):
    # what has left the window leaves the cache, and the tokens after it see what the prompt's do
    m = CacheMixer(64, heads=4, kv_heads=2, window=window, sinks=sinks, device=DEV)
    x = torch.randn((2, 150, 64), device=DEV).half()
    pos = grid_positions(1, 10, 15, device=DEV)
    want = f64(m(x, pos))
    cache = m.new_cache(capacity, batch=2, page_size=8)
    lengths = torch.tensor([4, 1], dtype=torch.int32, device=DEV)
    m(x[:, :4].contiguous(), pos[:4], cache, lengths)
    y = torch.stack([m.step(torch.stack([x[0, 4 + t], x[1, 1 + t]]), pos[4 + t:5 + t], cache) for t in range(146)])
    torch.cuda.synchronize()
    assert rms(y[:, 0], want[0, 4:]) <= 16 * U[torch.float16]
    assert cache.most <= capacity and cache.lengths.tolist()[0] <= capacity and bool((cache.mass == 0).all())
    # the other stream is three tokens behind, with the positions of the first
    alone = m.new_cache(capacity, page_size=8)
    m(x[1:, :1].contiguous(), pos[:1], alone)
    z = torch.cat([m.step(x[1:, 1 + t], pos[4 + t:5 + t], alone) for t in range(146)])
    assert rms(y[:, 1], f64(z)) <= 16 * U[torch.float16]


def test_a_budget_holds_the_first_the_latest_and_the_heaviest():
    m = CacheMixer(64, heads=4, kv_heads=2, sinks=3, device=DEV)
    full = m.new_cache(200)
    cache = m.new_cache(64, keep=40, recent=8)
    x = torch.randn((200, 1, 64), device=DEV).half()
    pos = grid_positions(1, 10, 20, device=DEV)
    for t in range(200):
        a, b = m.step(x[t], pos[t:t + 1], full), m.step(x[t], pos[t:t + 1], cache)
        if t < 64:
            assert torch.equal(a, b)  # nothing has been cut yet
        assert cache.most == int(cache.lengths[0]) <= 64 and torch.isfinite(b).all()
    # the first tokens are in their places still
    k, v = (y[full.table[0, 0].long(), :3] for y in (full.k, full.v))
    assert torch.equal(cache.k[cache.table[0, 0].long(), :3], k) and torch.equal(cache.v[cache.table[0, 0].long(), :3], v)
    # and the latest: position 199 of the stream
    n = int(cache.lengths[0]) - 1
    assert torch.equal(cache.k[cache.table[0, n // 16].long(), n % 16], full.k[full.table[0, 199 // 16].long(), 199 % 16])
    # weights of the held tokens: each step gave out one for every head
    assert float(cache.mass.sum()) > 0 and bool((cache.mass[..., n + 1:64] == 0).all())


def test_beside_the_encoder_and_the_decoder():
    flat = synth.make_weights(64, 2, 2)
    enc, dec = (Codec(64, 64, 64, 2, 2, "fp16", flat, device=DEV) for _ in range(2))
    m = CacheMixer(64, sinks=2, device=DEV)
    ce, cd = (m.new_cache(40, keep=20, recent=4) for _ in range(2))
    for t, frame in enumerate(synth.frame_sequence("tiny")):
        q, _ = enc.encode(torch.from_numpy(frame).to(DEV))
        dec.decode(q)
        a, b = m.frame(enc.get_state()[1], t, ce), m.frame(dec.get_state()[1], t, cd)
        torch.cuda.synchronize()
        assert a.shape == (64, 4, 4) and torch.equal(a, b) and torch.equal(ce.mass, cd.mass)


def test_command(capsys):
    main()
    assert "over the cache" in capsys.readouterr().out


def test_refusals():
    m = CacheMixer(64, device=DEV)
    x, pos = torch.randn((1, 8, 64), device=DEV).half(), grid_positions(1, 2, 4, device=DEV)
    cache = m.new_cache(8)
    m(x, pos, cache)
    with pytest.raises(ValueError, match="empty"):
        m(x, pos, cache)
    with pytest.raises(ValueError, match="fit"):
        m.step(x[:, 0], pos[:1], cache)
    with pytest.raises(ValueError):
        TokenCache(1, 8, 1, 64, keep=8)
    with pytest.raises(ValueError):
        CacheMixer(64, window=4, device=DEV).new_cache(8, keep=4)
    with pytest.raises(ValueError, match="fit"):
        m(torch.randn((1, 20, 64), device=DEV).half(), grid_positions(1, 4, 5, device=DEV), m.new_cache(16, keep=8))


def test_an_append_that_is_refused_leaves_the_cache_as_it_was():
    cache = TokenCache(2, 16, 1, 64, keep=8, sinks=1, recent=2, device=DEV)
    x = torch.randn((2, 14, 1, 64), device=DEV).half()
    cache.append(x[:, :12], x[:, :12])
    for tokens in (9, 14):
        with pytest.raises(ValueError, match="fit"):
            cache.append(x[:, :tokens], x[:, :tokens])
        assert cache.most == 12 and cache.lengths.tolist() == [12, 12]
    cache.append(x[:, :8], x[:, :8])
    assert cache.most == 16 and cache.lengths.tolist() == [16, 16]
