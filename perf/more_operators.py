"""The operators of exact attention over latent tokens whose speed is looked after: a prompt, a paged cache, its upkeep.

A token is one position of the 1/16 latent grid, (frame, row, column); a 64 x 64 frame has 16 of them, 480 x 832
1560, 1080p 8160 and 4K 32640 (136 rows of 240).  Token i sees the tokens j <= i with i - j < window or j < sinks
(window 0: all of them).  An encoder has all tokens of a frame or clip at once, a decoder has them one by one and
keeps keys and values in a cache of pages.  Each case is one pass through one operator of
``paper_2502_20762_amd.tokens``:

  window   softmax attention over whole sequences, with a sliding window and sinks
  paged    one new token of each sequence over its cached keys and values, with the weights summed up where wanted
  append   keys and values of new tokens into the pages of the cache
  evict    the heaviest tokens of each sequence and head, the first and the latest, copied to fewer pages

``run`` computes an operator in plain float32 torch operations, or, where ``own`` is true, through the package.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases
def _window(name, batch, tokens, heads, kv_heads, dim, vdim, dtype, window=0, sinks=0, ragged=False, layout="packed"):
    return {"name": name, "op": "window", "batch": batch, "tokens": tokens, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "vdim": vdim, "dtype": dtype, "window": window, "sinks": sinks, "ragged": ragged,
            "layout": layout}


def _paged(name, batch, tokens, heads, kv_heads, dim, vdim, dtype, page, window=0, sinks=0, ragged=False, mass=False):
    return {"name": name, "op": "paged", "batch": batch, "tokens": tokens, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "vdim": vdim, "dtype": dtype, "page": page, "window": window, "sinks": sinks, "ragged": ragged,
            "mass": mass}


def _append(name, batch, tokens, kv_heads, dim, vdim, dtype, page, before=0, ragged=False, mass=False):
    return {"name": name, "op": "append", "batch": batch, "tokens": tokens, "kv_heads": kv_heads, "dim": dim,
            "vdim": vdim, "dtype": dtype, "page": page, "before": before, "ragged": ragged, "mass": mass}


def _evict(name, batch, tokens, kv_heads, dim, vdim, dtype, page, keep, sinks, recent, ragged=False):
    return {"name": name, "op": "evict", "batch": batch, "tokens": tokens, "kv_heads": kv_heads, "dim": dim,
            "vdim": vdim, "dtype": dtype, "page": page, "keep": keep, "sinks": sinks, "recent": recent,
            "ragged": ragged}


def listed():
    return [
        # a thumbnail's frame as a prompt: a launch and little else
        _window("window_tiny_frame", 1, 16, 8, 8, 64, 64, "fp16"),
        # eight streams of WVGA frames of different fill (one empty, one a single token), every earlier token seen
        _window("window_wvga_ragged", 8, 1560, 8, 2, 64, 96, "bf16", ragged=True),
        # a 1080p frame, each token seeing the half frame before it and the first 64 tokens
        _window("window_hd1080", 1, 8160, 8, 8, 64, 64, "fp16", window=4080, sinks=64),
        # a 4K frame with wide heads, a quarter of the frame and its first row in sight: the largest products
        _window("window_uhd4k", 1, 32640, 16, 4, 128, 128, "bf16", window=8160, sinks=240, layout="heads"),
        # one stream's next token early in a small frame: latency
        _paged("paged_token", 1, 200, 8, 8, 64, 64, "fp16", 16),
        # the next token of 64 streams that are 1080p frames of different fill, shared key heads
        _paged("paged_streams", 64, 8160, 16, 4, 128, 128, "bf16", 64, ragged=True),
        # the next token of one stream after a clip of four 4K frames: few rows, a long cache
        _paged("paged_clip", 1, 130560, 16, 4, 128, 128, "fp16", 256),
        # eight streams, half a 1080p frame in sight, the weights summed for a later eviction
        _paged("paged_mass", 8, 8160, 8, 8, 64, 64, "fp16", 32, window=4080, sinks=64, mass=True),
        # one token of 64 streams into the cache
        _append("append_step", 64, 1, 8, 64, 64, "fp16", 16, before=1560, mass=True),
        # a clip of four 4K frames into the cache: the largest copy
        _append("append_clip", 1, 130560, 4, 128, 128, "bf16", 256),
        # 64 streams cut back to half of what they hold, each head by its own weights
        _evict("evict_streams", 64, 2040, 8, 64, 64, "fp16", 16, 1020, 16, 240, ragged=True),
        # one long stream, from four 4K frames' tokens to one
        _evict("evict_clip", 1, 130560, 4, 128, 128, "bf16", 256, 32640, 240, 8160),
    ]


def _log(rng, lo, hi):
    return min(max(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))), lo), hi)


def draw(rng):
    """A case of the same ranges: one token to a clip, narrow to wide, even and odd sizes, each type, layout and option."""
    op = rng.choice(["window", "paged", "append", "evict"])
    dtype = rng.choice(["fp16", "bf16"])
    while True:
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4])
        dim = rng.choice([16, 32, 64, 64, 96, 128, 128, 40, 75])
        vdim = rng.choice([dim, dim, 32, 64, 128, 33])
        page = rng.choice([16, 16, 32, 64, 128, 256])
        ragged = rng.random() < 0.4
        batch = _log(rng, 1, 64)
        if op == "window":
            tokens = _log(rng, 2, 32640)
            window = 0 if rng.random() < 0.3 else _log(rng, 1, 8160)
            sinks = rng.choice([0, 1, 4, 64, 240])
            c = _window("", batch, tokens, heads, kv, dim, vdim, dtype, window, sinks, ragged,
                        rng.choice(["packed", "heads"]))
            # no more pairs than the largest listed case has, a whole square where all earlier tokens are seen
            pairs = tokens * (min(window + sinks, tokens) if window else tokens)
            ok = batch * heads * pairs * (max(dim, 64) + max(vdim, 64)) <= 16 * 32640 * 8160 * 256
            ok = ok and batch * heads * tokens <= 16 * 32640
        elif op == "paged":
            tokens = _log(rng, 1, 130560)
            window = 0 if rng.random() < 0.6 else _log(rng, 1, 16384)
            c = _paged("", batch, tokens, heads, kv, dim, vdim, dtype, page, window, rng.choice([0, 1, 4, 64, 240]),
                       ragged, rng.random() < 0.3)
            ok = batch * tokens * kv * (dim + vdim) <= 64 * 8160 * 4 * 256 and batch * tokens * heads <= 64 * 8160 * 16
        elif op == "append":
            tokens = 1 if rng.random() < 0.3 else _log(rng, 2, 130560)
            c = _append("", batch, tokens, kv, dim, vdim, dtype, page, rng.choice([0, 1, 77, 1560, 8160]), ragged,
                        rng.random() < 0.5)
            ok = batch * tokens * kv * (dim + vdim) <= 130560 * 4 * 256 and batch * (tokens + c["before"]) * kv <= 1 << 21
        else:
            tokens = _log(rng, 64, 130560)
            keep = max(8, round(tokens * rng.uniform(0.1, 0.9)))
            sinks = min(rng.choice([0, 1, 4, 16, 240]), keep // 4)
            recent = min(rng.choice([0, 1, 64, 240, 8160]), keep // 2)
            c = _evict("", batch, tokens, kv, dim, vdim, dtype, page, keep, sinks, recent, ragged)
            ok = batch * keep * kv * (dim + vdim) <= 64 * 1020 * 8 * 128 and batch * tokens * kv <= 64 * 2040 * 8
        if ok:
            del c["name"]
            return c


def _lengths(c):
    """Tokens of each sequence: all of them, or for a ragged batch full, empty, one token, and between."""
    B, T = c["batch"], c["tokens"]
    if not c["ragged"]:
        return [T] * B
    return [(T, 0, 1)[b] if b < 3 else (b * 2654435761 >> 7) % (T + 1) for b in range(B)]


def _seen(c, i):
    """How many tokens token i sees."""
    W = c["window"] or i + 1
    return min(i + 1, W) + min(c["sinks"], max(0, i + 1 - W))


def work(c):
    op, K, D, V = c["op"], c["kv_heads"], c["dim"], c["vdim"]
    lengths, B = _lengths(c), c["batch"]
    tokens = sum(lengths)
    if op == "window":
        H = c["heads"]
        upto = [0]  # pairs of a sequence of so many tokens
        for i in range(c["tokens"]):
            upto.append(upto[-1] + _seen(c, i))
        # padding is not read, but its outputs are written as zeros
        return {"bytes": 2 * (tokens * (H * D + K * D + K * V) + B * c["tokens"] * H * V),
                "flops": 2 * (D + V) * H * sum(upto[n] for n in lengths)}
    if op == "paged":
        H, seen = c["heads"], sum(_seen(c, n - 1) for n in lengths if n)
        return {"bytes": 2 * (seen * K * (D + V) + B * H * (D + V)) + 4 * seen // c["page"] + (8 * seen * K if c["mass"] else 0),
                "flops": 2 * (D + V) * H * seen}
    if op == "append":
        return {"bytes": 4 * tokens * K * (D + V) + (4 * tokens * K if c["mass"] else 0), "flops": 0}
    kept = sum(min(n, c["keep"]) for n in lengths)
    # the weights of all, the kept rows in and out, and for every place of the result a weight and a position
    return {"bytes": 4 * tokens * K + 4 * kept * K * (D + V) + 8 * B * c["keep"] * K, "flops": 0}


# ---------------------------------------------------------------- inputs
def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    op, B, T, K, D, V = c["op"], c["batch"], c["tokens"], c["kv_heads"], c["dim"], c["vdim"]

    def randn(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(dt)

    s = {"case": c}
    lengths = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    if op == "window":
        H = c["heads"]
        if c["layout"] == "packed" and D == V:  # views of one projection's output: queries, keys, values of each token
            qkv = randn(B, T, H + 2 * K, D)
            s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:]
        elif c["layout"] == "packed":
            s["q"], s["k"], s["v"] = randn(B, T, H, D), randn(B, T, K, D), randn(B, T, K, V)
        else:
            s["q"], s["k"], s["v"] = (randn(B, h, T, d).transpose(1, 2) for h, d in ((H, D), (K, D), (K, V)))
        # queries and keys as a norm leaves them, some of the directions in common: a few tokens weigh most
        s["q"] += randn(1, 1, 1, D)
        s["k"] += randn(1, 1, 1, D, scale=0.5)
        s["lengths"] = lengths if c["ragged"] else None
        return s

    page = c["page"]

    def pages(tokens, first, spare=3):
        """A table of pages for so many tokens of each sequence, in no order, and how many pages that takes."""
        per = -(-tokens // page)
        ids = torch.randperm(B * per + spare, generator=g, device=DEV)[:B * per] + first
        return ids.reshape(B, per).to(torch.int32).contiguous(), first + B * per + spare

    capacity = T + c.get("before", 0)
    s["table"], count = pages(capacity, 0)
    if op == "evict":
        s["new_table"], count = pages(c["keep"], count)
    s["k_cache"], s["v_cache"] = randn(count, page, K, D), randn(count, page, K, V)
    columns = s["table"].shape[1] * page
    if op == "append":
        s["k"], s["v"] = randn(B, T, K, D), randn(B, T, K, V)
        s["starts"] = torch.full((B,), c["before"], dtype=torch.int32, device=DEV)
        s["counts"] = lengths if c["ragged"] else None
        s["mass"] = torch.rand((B, K, columns), generator=g, device=DEV) if c["mass"] else None
        return s
    s["lengths"] = lengths
    # summed weights: most tokens hardly any, a few much, and some none at all
    mass = torch.rand((B, K, columns), generator=g, device=DEV).reciprocal_().sub_(1.0)
    mass[torch.rand((B, K, columns), generator=g, device=DEV) < 0.05] = 0.0
    if op == "evict":
        s["mass"] = mass
        return s
    s["q"] = randn(B, c["heads"], D, scale=1.5)
    s["mass"] = mass if c["mass"] else None
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        from paper_2502_20762_amd import tokens
        if op == "window":
            return tokens.window_attention(s["q"], s["k"], s["v"], window=c["window"] or None, sinks=c["sinks"],
                                           lengths=s["lengths"])
        if op == "paged":
            o = tokens.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"],
                                       window=c["window"] or None, sinks=c["sinks"], mass=s["mass"])
            return (o, s["mass"]) if c["mass"] else o
        if op == "append":
            tokens.cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["starts"],
                                counts=s["counts"], mass=s["mass"])
            return (s["k_cache"], s["v_cache"], s["mass"]) if c["mass"] else (s["k_cache"], s["v_cache"])
        lengths, mass, kept = tokens.cache_evict(s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["mass"],
                                                 c["keep"], s["new_table"], sinks=c["sinks"], recent=c["recent"])
        return s["k_cache"], s["v_cache"], lengths, mass, kept
    return {"window": _plain_window, "paged": _plain_paged, "append": _plain_append, "evict": _plain_evict}[op](s)


def _plain_window(s):
    """Blocks of queries, each over the keys of its own block and of the window before it, and over the sinks."""
    c = s["case"]
    B, T, H, K, D, V = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["vdim"]
    G, dt = H // K, s["q"].dtype
    before = c["window"] if 0 < c["window"] < T else 0  # keys before a block
    L = min(T, max(64, -(-before // 4))) if before else T
    n = -(-T // L)

    def padded(x, front):  # (B, T, heads, d) -> (B, heads, front + n L, d) in 32 bits, zeros around
        y = x.float().transpose(1, 2)
        return torch.cat([y.new_zeros(*y.shape[:2], front, y.shape[3]), y,
                          y.new_zeros(*y.shape[:2], n * L - T, y.shape[3])], 2)

    q = padded(s["q"], 0).mul_(D ** -0.5).reshape(B, K, G, n, L, D).transpose(2, 3)  # (B, K, n, G, L, D)
    k, v = (padded(s[x], before).unfold(2, before + L, L) for x in "kv")  # (B, K, n, d, keys)
    i = torch.arange(n * L, device=DEV).reshape(n, L, 1)
    j = (L * torch.arange(n, device=DEV)[:, None] - before + torch.arange(before + L, device=DEV)).reshape(n, 1, -1)
    seen = (j <= i) & (j >= 0)
    S = min(c["sinks"], T) if before else 0
    if before:
        seen &= i - j < c["window"]
    if S:  # the sinks that the window has left behind
        seen = torch.cat([torch.arange(S, device=DEV) <= i - c["window"], seen], 2)
        k = torch.cat([s["k"][:, :S].float().permute(0, 2, 3, 1)[:, :, None].expand(B, K, n, D, S), k], 4)
        v = torch.cat([s["v"][:, :S].float().permute(0, 2, 3, 1)[:, :, None].expand(B, K, n, V, S), v], 4)
    p = torch.matmul(q.reshape(B * K * n, G * L, D), k.reshape(B * K * n, D, -1)).reshape(B, K, n, G, L, -1)
    p = p.masked_fill_(~seen[:, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    v = v.transpose(3, 4).reshape(B * K * n, -1, V)
    o = torch.matmul(p.reshape(B * K * n, G * L, -1), v).reshape(B, K, n, G, L, V) / total
    o = o.permute(0, 2, 4, 1, 3, 5).reshape(B, n * L, H, V)[:, :T]
    if s["lengths"] is not None:
        live = torch.arange(T, device=DEV) < s["lengths"][:, None]
        o = torch.where(live[:, :, None, None], o, 0.0)
    return o.to(dt)


def _plain_paged(s):
    c = s["case"]
    B, H, K, D, V = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["vdim"]
    G, table = H // K, s["table"].long()
    k = s["k_cache"][table].float().reshape(B, -1, K, D).permute(0, 2, 3, 1)  # (B, K, D, columns)
    v = s["v_cache"][table].float().reshape(B, -1, K, V).transpose(1, 2)
    j = torch.arange(k.shape[3], device=DEV)
    n = s["lengths"][:, None]
    seen = j < n
    if c["window"]:
        seen &= (j >= n - c["window"]) | (j < c["sinks"])
    p = torch.matmul(s["q"].float().reshape(B, K, G, D), k).mul_(D ** -0.5)
    p = p.masked_fill_(~seen[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    o = o.reshape(B, H, V).to(s["q"].dtype)
    if not c["mass"]:
        return o
    s["mass"] += (p / torch.where(total > 0, total, 1.0)).sum(2)
    return o, s["mass"]


def _plain_append(s):
    c = s["case"]
    T, page = c["tokens"], c["page"]
    at = s["starts"].long()[:, None] + torch.arange(T, device=DEV)
    p, r = s["table"].long().gather(1, at // page), at % page
    k, v = s["k"], s["v"]
    new = None
    if s["counts"] is not None:  # the rows of tokens that are not there keep what they hold
        new = torch.arange(T, device=DEV) < s["counts"][:, None]
        k = torch.where(new[:, :, None, None], k, s["k_cache"][p, r])
        v = torch.where(new[:, :, None, None], v, s["v_cache"][p, r])
    s["k_cache"][p, r] = k
    s["v_cache"][p, r] = v
    if s["mass"] is None:
        return s["k_cache"], s["v_cache"]
    to = at[:, None].expand(-1, c["kv_heads"], -1)
    s["mass"].scatter_(2, to, 0.0 if new is None else torch.where(new[:, None], 0.0, s["mass"].gather(2, to)))
    return s["k_cache"], s["v_cache"], s["mass"]


def _plain_evict(s):
    c = s["case"]
    B, K, page, keep = c["batch"], c["kv_heads"], c["page"], c["keep"]
    mass, n = s["mass"], s["lengths"].long()[:, None, None]
    j = torch.arange(mass.shape[2], device=DEV)
    rank = torch.where((j < c["sinks"]) | (j >= n - c["recent"]), math.inf, mass)
    rank = torch.where(j < n, rank, -math.inf)
    first = torch.sort(rank, dim=2, descending=True, stable=True).indices[..., :keep]
    kept = torch.where(first < n, first, mass.shape[2]).sort(2).values  # in order of position, none at the end
    new = kept < n
    old = torch.where(new, kept, 0)
    b = torch.arange(B, device=DEV)[:, None, None]
    h = torch.arange(K, device=DEV)[:, None]
    to = torch.arange(keep, device=DEV)
    p, r = s["table"].long()[b, old // page], old % page
    q, t = s["new_table"].long()[:, to // page][:, None], to % page
    for x in ("k_cache", "v_cache"):
        s[x][q, t, h] = torch.where(new[..., None], s[x][p, r, h], s[x][q, t, h])
    new_mass = mass.new_zeros(B, K, s["new_table"].shape[1] * page)
    new_mass[..., :keep] = torch.where(new, mass.gather(2, old), 0.0)
    return (s["k_cache"], s["v_cache"], n.flatten().clamp(max=keep).to(torch.int32), new_mass,
            torch.where(new, kept, -1).to(torch.int32))


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    return {"window": _exact_window, "paged": _exact_paged, "append": _exact_append, "evict": _exact_evict}[c["op"]](c, s)


def _exact_window(c, s):
    """A sequence and a stretch of queries at a time, with the list of the tokens that any of them sees."""
    B, T, H, V = c["batch"], c["tokens"], c["heads"], c["vdim"]
    group = H // c["kv_heads"]
    W = c["window"] or T
    out = torch.zeros(B, T, H, V, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(c)):
        for a in range(0, n, 512):
            e = min(n, a + 512)
            near = max(0, a - W + 1)
            j = torch.cat([torch.arange(min(c["sinks"], near)), torch.arange(near, e)]).to(DEV)
            i = torch.arange(a, e, device=DEV)[:, None]
            hidden = (j > i) | ((i - j >= W) & (j >= c["sinks"]))
            K, X = (s[x][b].index_select(0, j).double().transpose(0, 1).repeat_interleave(group, 0) for x in "kv")
            z = torch.matmul(s["q"][b, a:e].double().transpose(0, 1), K.transpose(1, 2).contiguous()) / math.sqrt(c["dim"])
            z[:, hidden] = -math.inf
            out[b, a:e] = torch.matmul(torch.softmax(z, -1), X).transpose(0, 1)
    return out


def _seen_positions(c, n):
    W = c["window"] or n
    near = max(0, n - W)
    return torch.cat([torch.arange(min(c["sinks"], near)), torch.arange(near, n)]).to(DEV)


def _exact_paged(c, s):
    B, H, K, page = c["batch"], c["heads"], c["kv_heads"], c["page"]
    out = torch.zeros(B, H, c["vdim"], dtype=torch.float64, device=DEV)
    mass = s["mass"].double() if c["mass"] else None
    for b, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        j = _seen_positions(c, n)
        at = s["table"][b].long()[j // page], j % page
        for h in range(K):
            mine = slice(h * (H // K), (h + 1) * (H // K))
            k, v = s["k_cache"][at[0], at[1], h].double(), s["v_cache"][at[0], at[1], h].double()
            w = torch.softmax(torch.matmul(s["q"][b, mine].double(), k.t().contiguous()) / math.sqrt(c["dim"]), 1)
            out[b, mine] = torch.matmul(w, v)
            if c["mass"]:
                mass[b, h, j] += w.sum(0)
    return (out, mass) if c["mass"] else out


def _exact_append(c, s):
    page, K = c["page"], s["k_cache"].double()
    V, mass = s["v_cache"].double(), s["mass"].double() if c["mass"] else None
    for b, n in enumerate(_lengths(c)):
        at = torch.arange(c["before"], c["before"] + n, device=DEV)
        rows = s["table"][b].long()[at // page] * page + at % page
        K.flatten(0, 1).index_copy_(0, rows, s["k"][b, :n].double())
        V.flatten(0, 1).index_copy_(0, rows, s["v"][b, :n].double())
        if c["mass"]:
            mass[b, :, c["before"]:c["before"] + n] = 0.0
    return (K, V, mass) if c["mass"] else (K, V)


def _exact_evict(c, s):
    page, keep = c["page"], c["keep"]
    K, V, mass = s["k_cache"].double(), s["v_cache"].double(), s["mass"].cpu().numpy()
    lengths, new_mass = [], np.zeros((c["batch"], c["kv_heads"], s["new_table"].shape[1] * page))
    kept = np.full((c["batch"], c["kv_heads"], keep), -1, np.int32)
    for b, n in enumerate(_lengths(c)):
        m = min(n, keep)
        lengths.append(m)
        for h in range(c["kv_heads"]):
            w = mass[b, h, :n].astype(np.float64)
            fixed = np.arange(n)
            fixed = (fixed < c["sinks"]) | (fixed >= n - c["recent"])
            order = np.lexsort((np.arange(n), -w, ~fixed))  # the fixed ones, then by weight, then by position
            got = np.sort(order[:m])
            kept[b, h, :m], new_mass[b, h, :m] = got, w[got]
            old = torch.from_numpy(got).to(DEV)
            to = torch.arange(m, device=DEV)
            src = s["table"][b].long()[old // page], old % page
            dst = s["new_table"][b].long()[to // page], to % page
            K[dst[0], dst[1], h] = s["k_cache"][src[0], src[1], h].double()
            V[dst[0], dst[1], h] = s["v_cache"][src[0], src[1], h].double()
    return K, V, torch.tensor(lengths, dtype=torch.int32), torch.from_numpy(new_mass), torch.from_numpy(kept)
