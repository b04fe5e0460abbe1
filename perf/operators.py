"""The operators around a cache of keys and values in 4 bits: what is timed, in plain torch and through the package.

Five operators of a serving step, on requests of different lengths that share one paged cache:

  tables   from the requests' lengths: pages from a free list, the slot and the position of every new token
  rope     rotary positions of a [tokens, heads, head_dim] tensor (both layouts, part of the head, both directions)
  append   rotary positions of the queries and keys, keys and values stored in 4 bits at the tokens' slots; the stored
           rows are read back ("read") as the numbers they stand for
  attend   attention of the new tokens over the cache: causal, or a sliding window with a few first tokens that stay visible

The cache holds, per page and key/value head, blocks of 16 tokens (head_dim rounded up to W = 64, 128 or 256):

  16 * W/2 bytes   key codes, [token][W/2], two e2m1 codes a byte, the lower dimension in the low half
  16 * W/2 bytes   value codes, [stretch of W/8 dimensions][token][W/16], each stretch's bytes XORed as in `_v_order`
  16 * W/16 bytes  key scales (e4m3, one for 16 dimensions), [token][W/16]
  16 * W/16 bytes  value scales, [W/16][token]

A number is code * scale * k_scale (or v_scale).
"""
import math

import torch

own = False

DEV = "cuda"
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
K_SCALE, V_SCALE = 1 / 32, 73 / 4096     # of a layer, exact in 32 bits
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decoding step's tables of a small batch: the latency of a launch
        {"name": "tables 16 decode", "op": "tables", "requests": 16, "new_low": 1, "new_high": 1, "ctx_low": 0, "ctx_high": 4000, "page": 16},
        # a mixed step: many requests, some with nothing new, some with a long prompt
        {"name": "tables 512 mixed", "op": "tables", "requests": 512, "new_low": 0, "new_high": 63, "ctx_low": 0, "ctx_high": 8000, "page": 64},
        # rotary positions of one decoding step
        {"name": "rope 16 half bf16", "op": "rope", "tokens": 16, "heads": 32, "head_dim": 128, "rope_dim": 128, "layout": "half", "inverse": False, "dtype": "bf16", "pad": 0},
        # the backward direction over a long sequence, a quarter of the head, neighbours as pairs, rows of a wider projection
        {"name": "rope 8191 pairs f32 back", "op": "rope", "tokens": 8191, "heads": 40, "head_dim": 96, "rope_dim": 24, "layout": "pairs", "inverse": True, "dtype": "f32", "pad": 64},
        # the new tokens of one decoding step enter the cache
        {"name": "append 16 bf16", "op": "append", "tokens": 16, "heads": 32, "kv_heads": 8, "head_dim": 128, "rope_dim": 128, "layout": "half", "page": 16, "dtype": "bf16"},
        # a prompt enters the cache
        {"name": "append 8192 bf16", "op": "append", "tokens": 8192, "heads": 32, "kv_heads": 8, "head_dim": 128, "rope_dim": 128, "layout": "half", "page": 64, "dtype": "bf16"},
        # the first steps of a single conversation: latency
        {"name": "attend 1x37", "op": "attend", "requests": 1, "new_low": 1, "new_high": 1, "len_low": 37, "len_high": 37, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 16, "window": 0, "sinks": 0, "dtype": "bf16"},
        # a serving batch of 16 conversations of different lengths, seven queries to a key/value head
        {"name": "attend 16x4000 ragged", "op": "attend", "requests": 16, "new_low": 1, "new_high": 1, "len_low": 100, "len_high": 4000, "heads": 28, "kv_heads": 4, "head_dim": 128,
         "page": 16, "window": 0, "sinks": 0, "dtype": "bf16"},
        # a large batch of long contexts: the cache's bytes count
        {"name": "attend 64x8192", "op": "attend", "requests": 64, "new_low": 1, "new_high": 1, "len_low": 8000, "len_high": 8192, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "window": 0, "sinks": 0, "dtype": "bf16"},
        # long contexts with a window and four first tokens, one head of queries to a head of keys, in 32 bits, four tokens at a time (drafts to be checked)
        {"name": "attend 8x32768 window f32", "op": "attend", "requests": 8, "new_low": 1, "new_high": 4, "len_low": 20000, "len_high": 32768, "heads": 16, "kv_heads": 16, "head_dim": 64,
         "page": 32, "window": 4096, "sinks": 4, "dtype": "f32"},
        # prompts of four requests, some behind a cached prefix
        {"name": "attend prompt 4x2048", "op": "attend", "requests": 4, "new_low": 1500, "new_high": 2048, "len_low": 2048, "len_high": 8192, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "window": 0, "sinks": 0, "dtype": "bf16"},
        # a prompt of odd sizes with a window, in 32 bits
        {"name": "attend prompt 700 f32", "op": "attend", "requests": 2, "new_low": 333, "new_high": 700, "len_low": 333, "len_high": 1500, "heads": 15, "kv_heads": 5, "head_dim": 80,
         "page": 16, "window": 501, "sinks": 3, "dtype": "f32"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("tables", "rope", "append", "attend", "attend", "attend"))
    page = rng.choice((16, 32, 64, 128))
    if op == "tables":
        n = _log(rng, 1, 512)
        return {"op": op, "requests": n, "new_low": rng.choice((0, 1)), "new_high": _log(rng, 1, max(1, 16384 // n)), "ctx_low": 0, "ctx_high": _log(rng, 1, 8000), "page": page}
    dim = rng.choice((64, 80, 96, 128, 128, 256))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    kv, group = rng.choice((1, 2, 4, 5, 8)), rng.choice((1, 2, 3, 4, 7, 8))
    if op in ("rope", "append"):
        rot, layout = rng.choice((dim, dim, dim // 2, dim // 4, 20)), rng.choice(("half", "pairs"))
        tokens = _log(rng, 1, 8192)
        tokens = max(1, min(tokens, 8192 * 40 * 96 // (kv * (group + 2) * dim)))
        if op == "rope":
            return {"op": op, "tokens": tokens, "heads": kv * group, "head_dim": dim, "rope_dim": rot, "layout": layout, "inverse": rng.random() < 0.5, "dtype": dtype, "pad": rng.choice((0, 8, 72))}
        return {"op": op, "tokens": tokens, "heads": kv * group, "kv_heads": kv, "head_dim": dim, "rope_dim": rot, "layout": layout, "page": page, "dtype": dtype}
    window, sinks = rng.choice(((0, 0), (0, 0), (_log(rng, 16, 4096), 0), (_log(rng, 16, 4096), rng.choice((1, 4, 21)))))
    case = {"op": op, "heads": kv * group, "kv_heads": kv, "head_dim": dim, "page": page, "window": window, "sinks": sinks, "dtype": dtype}
    n = _log(rng, 1, 64)
    if rng.random() < 0.6:      # single tokens, or a few
        new = rng.choice((1, 1, 1, 2, 5))
        high = _log(rng, max(16, new), 32768)
        high = max(new, min(high, 64 * 8192 * 8 * 128 // (n * kv * dim)))
        return {**case, "requests": n, "new_low": 1, "new_high": new, "len_low": max(new, _log(rng, 1, high)), "len_high": high}
    n = max(1, n // 8)
    new = _log(rng, 16, 2048)
    high = new + _log(rng, 1, 6144)
    most = 4 * 32 * 128 * 2048 * 5000 // (n * kv * group * dim)
    new = max(1, min(new, most // high))
    return {**case, "requests": n, "new_low": max(1, new // 3), "new_high": new, "len_low": new, "len_high": high}


def _spread(n, low, high):
    """n whole numbers from low to high that look drawn and are the same every time; the largest is among them."""
    return [high if i == n // 2 else low + int((i * 0.6180339887498949 % 1.0) * (high - low + 1)) for i in range(n)]


def _lengths(case):
    """(new tokens, keys) of each request of an attend case."""
    n = case["requests"]
    new = _spread(n, case["new_low"], case["new_high"])
    return new, [max(a, b) for a, b in zip(new, _spread(n, case["len_low"], case["len_high"])[::-1])]


def _width(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def _row_bytes(case):
    return _TYPES[case["dtype"]].itemsize * case["head_dim"]


def _kv_bytes(dim):
    """Codes and scales of one key or value row."""
    return dim / 2 + dim / 16


def _visible(case):
    """(pairs of a query and a key that it sees, keys that any query sees) over the requests."""
    w, s, pairs, keys = case["window"], case["sinks"], 0, 0
    for new, total in zip(*_lengths(case)):
        for p in range(total - new, total):
            low = max(0, p + 1 - w) if w else 0
            pairs += p + 1 - low + min(s, low)
        low = max(0, total - new + 1 - w) if w else 0
        keys += total - low + min(s, low)
    return pairs, keys


def work(case):
    op = case["op"]
    if op == "tables":
        n, t, p = case["requests"], sum(_spread(case["requests"], case["new_low"], case["new_high"])), case["page"]
        ctx = _spread(n, case["ctx_low"], case["ctx_high"])[::-1]
        new = _spread(n, case["new_low"], case["new_high"])
        fresh = sum(-(-(c + a) // p) - -(-c // p) for c, a in zip(ctx, new))
        # lengths, page numbers of new tokens, free pages taken; the tables' new entries, slots, positions, totals
        return {"bytes": 8 * n + 8 * fresh + 12 * t + 8 * n + 4 * n, "flops": 4 * t}
    if op == "rope":
        t, h, r = case["tokens"], case["heads"], case["rope_dim"]
        return {"bytes": 2 * t * h * _row_bytes(case) + t * (4 + 4 * r), "flops": 3 * t * h * r}
    if op == "append":
        t, h, kv, d, r = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"], case["rope_dim"]
        row = _row_bytes(case)
        # queries in and out, keys and values in, 4 bits out and in again, the rows read back
        return {"bytes": t * (2 * h * row + 2 * kv * row + 4 * kv * _kv_bytes(d) + 2 * kv * row + 12 + 4 * r), "flops": t * (3 * (h + kv) * r + 8 * kv * d)}
    pairs, keys = _visible(case)
    d = case["head_dim"]
    return {"bytes": 2 * sum(_lengths(case)[0]) * case["heads"] * _row_bytes(case) + 2 * keys * case["kv_heads"] * _kv_bytes(d), "flops": 4 * pairs * case["heads"] * d}


# ---------------------------------------------------------------------------------------------- the 4-bit cache, plainly

def _block_bytes(dim):
    return 16 * 2 * (_width(dim) // 2 + _width(dim) // 16)


def _v_order(width):
    """Where the value codes of a block of 16 tokens lie: [token, W/2] byte numbers."""
    vb = width // 16
    r, token, byte = torch.arange(8).view(8, 1, 1), torch.arange(16).view(1, 16, 1), torch.arange(vb).view(1, 1, vb)
    turned = {64: ((r >> 1) & 1) * 32, 128: (r & 1) * 64, 256: (r & 1) * 16}[width]
    return (r * 16 * vb + ((token * vb) ^ turned) + byte).permute(1, 0, 2).reshape(16, width // 2).to(DEV)


def _unpacked(codes, scales):
    """[..., W/2] bytes of two codes and [..., W/16] bytes of scales: the numbers [..., W] in 32 bits, before k_scale or v_scale."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEV)
    pair = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)
    return pair * scales.view(torch.float8_e4m3fn).float().repeat_interleave(16, -1)


def _rows_of(blocks, dim):
    """Blocks [..., block bytes]: keys and values [..., 16, dim] in 32 bits, before k_scale and v_scale."""
    w = _width(dim)
    part = blocks.split((8 * w, 8 * w, w, w), -1)
    k = _unpacked(part[0].unflatten(-1, (16, w // 2)), part[2].unflatten(-1, (16, w // 16)).contiguous())
    v = _unpacked(part[1][..., _v_order(w)], part[3].unflatten(-1, (w // 16, 16)).transpose(-1, -2).contiguous())
    return k[..., :dim], v[..., :dim]


def _quantised(x, scale):
    """Rows [..., dim] in 32 bits: (codes [..., W/2], scales [..., W/16]) as bytes."""
    w = _width(x.shape[-1])
    g = torch.nn.functional.pad(x, (0, w - x.shape[-1])).unflatten(-1, (w // 16, 16))
    s8 = (g.abs().amax(-1) * (1.0 / (6.0 * scale))).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = s8.float() * scale
    y = g * torch.where(s > 0, 1.0 / s, torch.zeros_like(s)).unsqueeze(-1)
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * (y < 0)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), s8.view(torch.uint8)


def _store(cache, k, v, slots, page, dim):
    """Rows of keys and values [T, heads, dim] in 32 bits into the cache [pages, heads, page/16, block bytes]."""
    w = _width(dim)
    (kc, ks), (vc, vs) = _quantised(k, K_SCALE), _quantised(v, V_SCALE)
    where, within = torch.div(slots, page, rounding_mode="floor"), slots % page
    token, head = within % 16, torch.arange(k.shape[1], device=DEV)
    at = (where.view(-1, 1, 1), head.view(1, -1, 1), torch.div(within, 16, rounding_mode="floor").view(-1, 1, 1))
    token, half, small = token.view(-1, 1, 1), torch.arange(w // 2, device=DEV).view(1, 1, -1), torch.arange(w // 16, device=DEV).view(1, 1, -1)
    cache[at + (token * (w // 2) + half,)] = kc
    cache[at + (8 * w + _v_order(w)[token.view(-1)].unsqueeze(1),)] = vc
    cache[at + (16 * w + token * (w // 16) + small,)] = ks
    cache[at + (17 * w + small * 16 + token,)] = vs


def _load(cache, slots, page, dim):
    """The keys and values at the slots, in 32 bits, [T, heads, dim]."""
    block = cache[torch.div(slots, page, rounding_mode="floor"), :, torch.div(slots % page, 16, rounding_mode="floor")]
    k, v = _rows_of(block, dim)
    token = (slots % 16).view(-1, 1, 1, 1).expand(-1, k.shape[1], 1, dim)
    return k.gather(2, token).squeeze(2) * K_SCALE, v.gather(2, token).squeeze(2) * V_SCALE


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _rows(g, t, heads, dim, dtype, pad=0):
    """[t, heads, dim] rows as a projection leaves them: some dimensions larger than others; `pad` elements of another tensor behind each token's heads."""
    loud = 1.0 + 3.0 * (torch.arange(dim, device=DEV) % 29 == 5)
    x = torch.empty((t, heads * dim + pad), dtype=dtype, device=DEV)
    x = x[:, : heads * dim].unflatten(1, (heads, dim))
    return x.copy_(_normal(g, t, heads, dim) * loud)


def _turns(n, rot):
    """cos and sin of position * 10000^(-2i/rot): [n, rot/2, 2] in 32 bits."""
    at = torch.arange(n, device=DEV, dtype=torch.float64).view(-1, 1) * 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    return torch.stack((at.cos(), at.sin()), -1).float()


def _cumulative(lengths):
    return torch.tensor([0] + lengths, device=DEV, dtype=torch.int32).cumsum(0, dtype=torch.int32)


def _plan(case, **more):
    from paper_2509_02753_b200 import kv_cache
    dtype = _TYPES[case.get("dtype", "bf16")]
    return kv_cache.KVPlan(n_heads=case.get("heads", 1), n_kv_heads=case.get("kv_heads", case.get("heads", 1)), head_dim=case.get("head_dim", 64),
                           page_size=case.get("page", 16), dtype=dtype, **more)


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    state = {"case": case}
    limits = {"max_requests": case.get("requests", 1), "max_tokens": 1}
    if op == "tables":
        n, p = case["requests"], case["page"]
        new, ctx = _spread(n, case["new_low"], case["new_high"]), _spread(n, case["ctx_low"], case["ctx_high"])[::-1]
        held = [-(-c // p) for c in ctx]
        width = max(-(-(c + a) // p) for c, a in zip(ctx, new)) + 1
        pool = torch.randperm(sum(held) + sum(-(-a // p) + 1 for a in new), generator=g, device=DEV, dtype=torch.int32)
        table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
        own_page = torch.arange(width, device=DEV) < torch.tensor(held, device=DEV).view(-1, 1)
        table[own_page] = pool[: sum(held)]
        state |= {"ctx": torch.tensor(ctx, dtype=torch.int32, device=DEV), "new": torch.tensor(new, dtype=torch.int32, device=DEV),
                  "free": pool[sum(held):].contiguous(), "table": table, "tokens": sum(new)}
        limits["max_tokens"] = max(1, sum(new))
    elif op == "rope":
        t = case["tokens"]
        state |= {"x": _rows(g, t, case["heads"], case["head_dim"], _TYPES[case["dtype"]], case["pad"]), "turns": _turns(max(t, 4096), case["rope_dim"]),
                  "positions": torch.randint(0, max(t, 4096), (t,), generator=g, device=DEV, dtype=torch.int32) if t < 64 else torch.arange(t, device=DEV, dtype=torch.int32)}
        limits["max_tokens"] = t
    elif op == "append":
        t, h, kv, d, p, dtype = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"], case["page"], _TYPES[case["dtype"]]
        n_pages = -(-t // p) + 7
        both = _rows(g, t, h + 2 * kv, d, dtype)      # one projection's output: queries, keys and values side by side
        turns = _turns(max(t, 4096), case["rope_dim"])
        if t < 64:      # a decoding step: every token in a page of its own request
            n_pages = t + 7
            page = torch.randperm(n_pages, generator=g, device=DEV)[:t]
            slots = page * p + torch.randint(0, p, (t,), generator=g, device=DEV)
            positions = torch.randint(0, 4096, (t,), generator=g, device=DEV, dtype=torch.int32)
        else:
            page = torch.randperm(n_pages, generator=g, device=DEV)
            at = torch.arange(t, device=DEV)
            slots, positions = page[at // p] * p + at % p, at.int()
        state |= {"q": both[:, :h], "k": both[:, h: h + kv], "v": both[:, h + kv:], "turns": turns, "slots": slots, "positions": positions,
                  "cache": torch.zeros((n_pages, kv, p // 16, _block_bytes(d)), dtype=torch.uint8, device=DEV)}
        limits["max_tokens"] = t
    else:
        n, h, kv, d, p, dtype = case["requests"], case["heads"], case["kv_heads"], case["head_dim"], case["page"], _TYPES[case["dtype"]]
        new, total = _lengths(case)
        width = -(-max(total) // p)
        held = torch.tensor([-(-a // p) for a in total], device=DEV)
        n_pages = int(held.sum()) + 3
        table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(width, device=DEV) < held.view(-1, 1)] = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int32)[:-3]
        # a store of quantised blocks of 16 tokens, from which every page takes its blocks
        store = torch.zeros((512, 1, 1, _block_bytes(d)), dtype=torch.uint8, device=DEV)
        some = _rows(g, 512 * 16, 2, d, torch.float32)
        _store(store, some[:, :1], some[:, 1:], torch.arange(512 * 16, device=DEV), 16, d)
        cache = store.view(512, -1)[torch.randint(0, 512, (n_pages * kv * (p // 16),), generator=g, device=DEV)].view(n_pages, kv, p // 16, -1)
        state |= {"q": _rows(g, sum(new), h, d, dtype), "cu": _cumulative(new), "len": torch.tensor(total, dtype=torch.int32, device=DEV), "table": table, "cache": cache,
                  "max_new": max(new), "longest": max(total)}
        limits["max_tokens"] = sum(new)
    if own:
        state["plan"] = _plan(case, **limits)
    return state


# ---------------------------------------------------------------------------------------------- the operators, plainly

def _tables(ctx, new, free, table, t, page):
    cu = torch.cat((torch.zeros(1, dtype=torch.int32, device=DEV), new.cumsum(0, dtype=torch.int32)))
    total = ctx + new
    held, wanted = (ctx + page - 1) // page, (total + page - 1) // page
    fresh = wanted - held
    first = fresh.cumsum(0, dtype=torch.int32) - fresh
    col = torch.arange(table.shape[1], device=DEV, dtype=torch.int32)
    mine = (col >= held.view(-1, 1)) & (col < wanted.view(-1, 1))
    at = (first.view(-1, 1) + col - held.view(-1, 1)).clamp(0, free.numel() - 1)
    table.copy_(torch.where(mine, free[at.long()], table))
    request = torch.searchsorted(cu[1:].contiguous(), torch.arange(t, device=DEV, dtype=torch.int32), right=True)
    positions = ctx[request] + torch.arange(t, device=DEV, dtype=torch.int32) - cu[request]
    slots = table[request, (positions // page).long()].long() * page + positions % page
    return total, cu, positions, slots, fresh.sum(0, keepdim=True, dtype=torch.int32)


def _rotated(x, turns, positions, rot, layout, inverse=False):
    """In 32 bits, not rounded."""
    x = x.float()
    cs = turns[positions.long()].unsqueeze(1)
    c, s = cs[..., 0], -cs[..., 1] if inverse else cs[..., 1]
    a, b = (x[..., : rot // 2], x[..., rot // 2: rot]) if layout == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    u, w = a * c - b * s, b * c + a * s
    turned = torch.cat((u, w), -1) if layout == "half" else torch.stack((u, w), -1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), -1)


def _attention(q, cu, lens, table, cache, longest, max_new, window, sinks, page):
    t, h, d = q.shape
    n, kv = lens.numel(), cache.shape[1]
    g = h // kv
    pages = table[:, : -(-longest // page)].clamp(min=0).long()
    k, v = _rows_of(cache[pages].transpose(1, 2), d)        # [n, kv, pages, page/16, 16, d]
    k, v = (x.flatten(2, 4)[:, :, :longest] for x in (k, v))
    new = (cu[1:] - cu[:-1]).view(-1, 1)
    row = torch.arange(max_new, device=DEV).view(1, -1)
    real = row < new
    source = (cu[:-1].view(-1, 1) + row).clamp(max=t - 1).long()
    qs = q[source].float().view(n, max_new, kv, g, d).permute(0, 2, 3, 1, 4).reshape(n, kv, g * max_new, d)
    s = torch.matmul(qs, k.transpose(-1, -2)).mul_(K_SCALE / math.sqrt(d)).view(n, kv, g, max_new, longest)
    key, p = torch.arange(longest, device=DEV).view(1, 1, -1), (lens.view(-1, 1) - new + row).unsqueeze(-1)
    see = key <= p
    if window:
        see = see & ((key > p - window) | (key < sinks))
    s.masked_fill_(~see.view(n, 1, 1, max_new, longest), -math.inf)
    top = s.amax(-1, keepdim=True)
    s = s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(n, kv, g * max_new, longest), v).mul_(V_SCALE).view(n, kv, g, max_new, d) / torch.where(total > 0, total, torch.ones_like(total))
    return o.permute(0, 3, 1, 2, 4).reshape(n, max_new, h, d)[real].to(q.dtype)


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        return _run_own(state, case, op)
    if op == "tables":
        total, cu, positions, slots, taken = _tables(state["ctx"], state["new"], state["free"], state["table"], state["tokens"], case["page"])
        return {"table": state["table"], "len": total, "cu": cu, "positions": positions, "slots": slots, "taken": taken}
    if op == "rope":
        return _rotated(state["x"], state["turns"], state["positions"], case["rope_dim"], case["layout"], case["inverse"]).to(state["x"].dtype)
    if op == "append":
        q, k = (_rotated(state[x], state["turns"], state["positions"], case["rope_dim"], case["layout"]) for x in "qk")
        _store(state["cache"], k, state["v"].float(), state["slots"], case["page"], case["head_dim"])
        k, v = _load(state["cache"], state["slots"], case["page"], case["head_dim"])
        return {"q": q.to(state["q"].dtype), "k": k.to(state["q"].dtype), "v": v.to(state["q"].dtype)}
    return _attention(state["q"], state["cu"], state["len"], state["table"], state["cache"], state["longest"], state["max_new"], case["window"], case["sinks"], case["page"])


def _run_own(state, case, op):
    plan = state["plan"]
    if op == "tables":
        total, cu, positions, slots, taken = plan.tables(state["ctx"], state["new"], state["free"], state["table"], state["tokens"])
        return {"table": state["table"], "len": total, "cu": cu, "positions": positions, "slots": slots, "taken": taken}
    if op == "rope":
        return plan.rope(state["x"], state["positions"], state["turns"], layout=case["layout"], inverse=case["inverse"])
    if op == "append":
        q = plan.append(state["q"], state["k"], state["v"], state["slots"], state["cache"], positions=state["positions"], turns=state["turns"], layout=case["layout"],
                        k_scale=K_SCALE, v_scale=V_SCALE)
        k, v = plan.read(state["cache"], state["slots"], k_scale=K_SCALE, v_scale=V_SCALE)
        return {"q": q, "k": k, "v": v}
    return plan.attention(state["q"], state["cu"], state["len"], state["table"], state["cache"], max_new=state["max_new"], window=case["window"], sinks=case["sinks"],
                          k_scale=K_SCALE, v_scale=V_SCALE)


# ---------------------------------------------------------------------------------------------- the operators' definitions in 64 bits

def _nearest(x, step):
    return torch.round(x / step) * step     # ties to the even multiple


def _exact_turned(x, angle, rot, layout, sign=1.0):
    """Rotation as a product of complex numbers."""
    x = x.double()
    at = torch.arange(rot // 2, device=DEV)
    at = (at, at + rot // 2) if layout == "half" else (2 * at, 2 * at + 1)
    z = torch.complex(x[..., at[0]], x[..., at[1]]) * torch.polar(torch.ones_like(angle), sign * angle).unsqueeze(1)
    y = x.clone()
    y[..., at[0]], y[..., at[1]] = z.real, z.imag
    return y


def _exact_stored(x, scale):
    """What a row stands for once it is held in 4 bits."""
    dim = x.shape[-1]
    g = torch.nn.functional.pad(x, (0, -dim % 16)).unflatten(-1, (-1, 16))
    t = g.abs().amax(-1, keepdim=True) / (6.0 * scale)
    s = _nearest(t, torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)).clamp(max=448.0) * scale
    a = torch.where(s > 0, g.abs() / s, torch.zeros_like(g))
    a = _nearest(a, torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))).clamp(max=6.0)
    return (a * s * g.sign()).flatten(-2)[..., :dim]


def _exact_decoded(block, dim):
    """Keys and values of blocks [m, block bytes], by the bits of a code: sign, two bits of exponent, one of fraction."""
    w, m = _width(dim), block.shape[0]

    def value(code):
        e, f = (code >> 1) & 3, code & 1
        a = torch.where(e == 0, 0.5 * f, (1 + 0.5 * f) * torch.exp2(e.double() - 1))
        return torch.where(code > 7, -a, a)

    def scale(byte):
        e, f = (byte >> 3) & 15, byte & 7
        return torch.where(e == 0, f * 2.0 ** -9, (1 + f / 8.0) * torch.exp2(e.double() - 7))

    b = block.int()
    d = torch.arange(dim, device=DEV).view(1, -1)
    t = torch.arange(16, device=DEV).view(-1, 1)
    r, within = d // (w // 8), (d % (w // 8)) // 2
    turned = ((r // 2) % 2) * 32 if w == 64 else (r % 2) * 64 if w == 128 else (r % 2) * 16
    at_k, at_v = t * (w // 2) + d // 2, 8 * w + r * w + ((t * (w // 16)) ^ turned) + within
    shift = 4 * (d % 2)
    k = value((b[:, at_k.flatten()].view(m, 16, dim) >> shift) & 15) * scale(b[:, (16 * w + t * (w // 16) + d // 16).flatten()].view(m, 16, dim))
    v = value((b[:, at_v.flatten()].view(m, 16, dim) >> shift) & 15) * scale(b[:, (17 * w + (d // 16) * 16 + t).flatten()].view(m, 16, dim))
    return k, v


def exact(case, seed):
    op = case["op"]
    if op == "tables":
        return None
    state = prepare(case, seed)
    d = case["head_dim"]
    if op in ("rope", "append"):
        angle = torch.atan2(state["turns"][..., 1].double(), state["turns"][..., 0].double())[state["positions"].long()]
        if op == "rope":
            return _exact_turned(state["x"], angle, case["rope_dim"], case["layout"], -1.0 if case["inverse"] else 1.0)
        q, k = (_exact_turned(state[x], angle, case["rope_dim"], case["layout"]) for x in "qk")
        return {"q": q, "k": _exact_stored(k, K_SCALE), "v": _exact_stored(state["v"].double(), V_SCALE)}
    new, total = _lengths(case)
    if 4.0 * _visible(case)[0] * case["heads"] * d > 3e12:
        return None
    h, kv, p, window, sinks = case["heads"], case["kv_heads"], case["page"], case["window"], case["sinks"]
    out, at = [], 0
    for i, (a, m) in enumerate(zip(new, total)):
        pages = state["table"][i, : -(-m // p)].long()
        query = torch.arange(m - a, m, device=DEV).view(-1, 1)
        key = torch.arange(m, device=DEV).view(1, -1)
        see = (key <= query) & ((query - key < window) | (key < sinks)) if window else key <= query
        heads = []
        for j in range(kv):
            k, v = (x.reshape(-1, d)[:m] for x in _exact_decoded(state["cache"][pages, j].flatten(0, 1), d))
            q = state["q"][at: at + a, j * (h // kv): (j + 1) * (h // kv)].double()
            s = torch.einsum("tgd,kd->gtk", q, k * K_SCALE) / math.sqrt(d)
            weight = torch.softmax(s.masked_fill(~see, -math.inf), -1)
            heads.append(torch.einsum("gtk,kd->tgd", weight, v * V_SCALE))
        out.append(torch.cat(heads, 1))
        at += a
    return torch.cat(out)
