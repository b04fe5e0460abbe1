"""Operators next to the attention over the 4-bit cache: what is timed, in plain torch and through the package.

A prefix that many requests share, and attention over the pages that a cheap score selects:

  prefix     groups of consecutive requests: how many leading pages their block tables have in common
  shared     attention of the new tokens over all their keys, those of a group's shared prefix read once for the group
  summarise  for every page that got new tokens, each dimension's largest and smallest stored key, in 8 bits; read back as numbers
  select     for every new token and key/value head the pages whose bounds promise the largest scores, the first and the
             last pages always among them
  selected   attention of the new tokens over the pages that are listed for them

The cache of keys and values in 4 bits holds, per page and key/value head, blocks of 16 tokens (head_dim rounded up to W = 64, 128 or 256):

  16 * W/2 bytes   key codes, [token][W/2], two e2m1 codes a byte, the lower dimension in the low half
  16 * W/2 bytes   value codes, [stretch of W/8 dimensions][token][W/16], each stretch's bytes XORed as in `_v_order`
  16 * W/16 bytes  key scales (e4m3, one for 16 dimensions), [token][W/16]
  16 * W/16 bytes  value scales, [W/16][token]

A number is code * scale * k_scale (or v_scale).  The summaries hold, per page and key/value head, 2 W + 16 bytes:

  W bytes          the largest keys as whole numbers of steps, rounded up (int8)
  W bytes          the smallest keys, rounded down
  4 bytes          the step (fp32; times k_scale), the largest magnitude / 127; 12 bytes of zeros
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
        # a small batch behind one system prompt: the latency of a launch
        {"name": "prefix 16", "op": "prefix", "requests": 16, "groups": 1, "prefix_low": 2000, "prefix_high": 2000, "own_low": 1, "own_high": 500, "new": 1, "page": 16},
        # a large batch over many prompts of different lengths
        {"name": "prefix 1000 in 37", "op": "prefix", "requests": 1000, "groups": 37, "prefix_low": 0, "prefix_high": 16000, "own_low": 1, "own_high": 3000, "new": 2, "page": 16},
        # a few conversations behind a short system prompt: latency
        {"name": "shared 8x512", "op": "shared", "requests": 8, "groups": 1, "prefix_low": 512, "prefix_high": 512, "own_low": 1, "own_high": 100, "new": 1,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16, "dtype": "bf16"},
        # a serving batch behind one long document
        {"name": "shared 64x8192", "op": "shared", "requests": 64, "groups": 1, "prefix_low": 8192, "prefix_high": 8192, "own_low": 1, "own_high": 500, "new": 1,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "dtype": "bf16"},
        # several samples of a few prompts, two tokens at a time (drafts to be checked), odd heads, in 32 bits
        {"name": "shared 45 in 4 f32", "op": "shared", "requests": 45, "groups": 4, "prefix_low": 900, "prefix_high": 5000, "own_low": 2, "own_high": 700, "new": 2,
         "heads": 15, "kv_heads": 5, "head_dim": 80, "page": 32, "dtype": "f32"},
        # one decoding step's tokens enter their pages' bounds
        {"name": "summarise 16 decode", "op": "summarise", "requests": 16, "new_low": 1, "new_high": 1, "len_low": 100, "len_high": 4000, "kv_heads": 8, "head_dim": 128, "page": 64},
        # prompts enter
        {"name": "summarise prompts 16384", "op": "summarise", "requests": 5, "new_low": 1000, "new_high": 5461, "len_low": 2000, "len_high": 9000, "kv_heads": 8, "head_dim": 128, "page": 64},
        # one conversation: latency
        {"name": "select 1x2000", "op": "select", "requests": 1, "new_low": 1, "new_high": 1, "len_low": 2000, "len_high": 2000, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 16, "n_select": 32, "first": 1, "last": 2, "dtype": "bf16"},
        # a serving batch of long contexts: the summaries' bytes count
        {"name": "select 64x32768", "op": "select", "requests": 64, "new_low": 1, "new_high": 1, "len_low": 20000, "len_high": 32768, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "n_select": 32, "first": 1, "last": 2, "dtype": "bf16"},
        # prompts of odd sizes, in 32 bits
        {"name": "select prompts 1500 f32", "op": "select", "requests": 3, "new_low": 333, "new_high": 1500, "len_low": 5000, "len_high": 16000, "heads": 14, "kv_heads": 2, "head_dim": 80,
         "page": 32, "n_select": 45, "first": 2, "last": 3, "dtype": "f32"},
        # a serving batch of long contexts, a sixteenth of each read
        {"name": "selected 16 of 32768", "op": "selected", "requests": 16, "new_low": 1, "new_high": 1, "len_low": 20000, "len_high": 32768, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 64, "n_select": 32, "first": 1, "last": 2, "dtype": "bf16"},
        # a prompt behind a long context, small pages, in 32 bits
        {"name": "selected prompt 500 f32", "op": "selected", "requests": 2, "new_low": 77, "new_high": 500, "len_low": 3000, "len_high": 6000, "heads": 14, "kv_heads": 2, "head_dim": 64,
         "page": 16, "n_select": 31, "first": 1, "last": 4, "dtype": "f32"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("prefix", "shared", "shared", "summarise", "select", "selected", "selected"))
    page = rng.choice((16, 32, 64, 128))
    dim = rng.choice((64, 80, 96, 128, 128, 256))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    kv, group = rng.choice((1, 2, 4, 5, 8)), rng.choice((1, 2, 3, 4, 7, 8))
    heads = {"heads": kv * group, "kv_heads": kv, "head_dim": dim, "page": page, "dtype": dtype}
    if op == "prefix":
        n = _log(rng, 1, 1000)
        high = _log(rng, 16, 16000)
        return {"op": op, "requests": n, "groups": _log(rng, 1, n), "prefix_low": rng.choice((0, high)), "prefix_high": high, "own_low": 1, "own_high": _log(rng, 1, 3000),
                "new": 1, "page": page}
    if op == "shared":
        n = _log(rng, 1, 64)
        new = rng.choice((1, 1, 2, 4))
        groups = min(n, rng.choice((1, 1, 1, 2, 5)))
        high = _log(rng, 64, 16384)
        high = min(high, 64 * 8192 * 32 * 128 // (n * new * kv * group * dim))
        return {"op": op, "requests": n, "groups": groups, "prefix_low": rng.choice((0, high // 2, high)), "prefix_high": high, "own_low": new,
                "own_high": new + _log(rng, 1, 700), "new": new, **heads}
    n = _log(rng, 1, 64)
    if op == "summarise":
        new = rng.choice((1, 1, 3, _log(rng, 16, max(16, 16384 // n))))
        return {"op": op, "requests": n, "new_low": max(1, new // 3), "new_high": new, "len_low": new, "len_high": new + _log(rng, 1, 4000), "kv_heads": kv, "head_dim": dim, "page": page}
    first, last = rng.choice((0, 1, 1, 3)), rng.choice((1, 2, 2, 5))
    most = _log(rng, first + last, 64)
    case = {"op": op, "n_select": most, "first": first, "last": last, **heads}
    if rng.random() < 0.6:      # single tokens, or a few
        new = rng.choice((1, 1, 1, 4))
        high = new + _log(rng, 16, 32768)
        high = max(new, min(high, 64 * 32768 * 8 * 128 // (n * kv * dim)))
        if op == "selected":
            high = max(new, min(high, 16 * 32768 * 8 * 128 // (n * kv * dim)))
    else:
        n = max(1, n // 8)
        new = _log(rng, 16, 1500)
        high = new + _log(rng, 16, 16000)
        if op == "selected":     # no more keys read than by the largest
            new = max(1, min(new, 64 * 32 * 64 * 8 * 128 // (n * most * page * kv * dim)))
        else:
            new = max(1, min(new, 64 * 512 * 8 * 128 * 32 // (n * (high // page + 1) * kv * dim)))
    return {**case, "requests": n, "new_low": max(1, new // 3), "new_high": new, "len_low": max(new, high // 2), "len_high": high}


def _spread(n, low, high):
    """n whole numbers from low to high that look drawn and are the same every time; the largest is among them."""
    return [high if i == n // 2 else low + int((i * 0.6180339887498949 % 1.0) * (high - low + 1)) for i in range(n)]


def _lengths(case):
    """(new tokens, keys) of each request."""
    n = case["requests"]
    new = _spread(n, case["new_low"], case["new_high"])
    return new, [max(a, b) for a, b in zip(new, _spread(n, case["len_low"], case["len_high"])[::-1])]


def _groups(case):
    """(first request of each group and the end, shared pages of each group, new tokens, keys of each request)."""
    n, g, p = case["requests"], case["groups"], case["page"]
    share = _spread(g, 1, 5)
    cu, at = [0], 0
    for i, s in enumerate(share):
        at += s
        cu.append(n if i == g - 1 else max(cu[-1] + 1, min(n - (g - 1 - i), at * n // sum(share))))
    pages = [x // p for x in _spread(g, case["prefix_low"], case["prefix_high"])]
    behind = _spread(n, case["own_low"], case["own_high"])
    total = [0] * n
    for j in range(g):
        for i in range(cu[j], cu[j + 1]):
            total[i] = pages[j] * p + max(behind[i], case["new"])
    return cu, pages, [case["new"]] * n, total


def _width(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def _row_bytes(case):
    return _TYPES[case["dtype"]].itemsize * case["head_dim"]


def _kv_bytes(dim):
    """Codes and scales of one key or value row."""
    return dim / 2 + dim / 16


def _listed_pages(p, case):
    """Pages that a token at position p reads."""
    return min(p // case["page"] + 1, case["n_select"])


def work(case):
    op, p = case["op"], case["page"]
    if op in ("prefix", "shared"):
        cu, pages, new, total = _groups(case)
        sizes = [b - a for a, b in zip(cu, cu[1:])]
        if op == "prefix":
            # the tables' leading entries, lengths; the groups' and requests' answers
            cells = sum(m * (s + 1) for m, s in zip(sizes, pages) if m > 1)
            return {"bytes": 4 * cells + 4 * len(cu) + 8 * case["requests"] + 4 * (case["groups"] + case["requests"]), "flops": cells}
        h, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
        pairs = sum(t - a + j + 1 for a, t in zip(new, total) for j in range(a))
        keys = sum(pages) * p + sum(total) - sum(m * s * p for m, s in zip(sizes, pages))
        return {"bytes": 2 * sum(new) * h * _row_bytes(case) + 2 * keys * kv * _kv_bytes(d), "flops": 4 * pairs * h * d}
    new, total = _lengths(case)
    kv, d = case["kv_heads"], case["head_dim"]
    if op == "summarise":
        touched = [(a, t - (t - a) // p * p, -(-t // p) - (t - a) // p) for a, t in zip(new, total)]
        keys, pages = sum(k for _, k, _ in touched), sum(m for _, _, m in touched)
        # keys of the touched pages; their bounds out and in again, and as numbers
        return {"bytes": kv * (keys * _kv_bytes(d) + pages * (2 * (2 * d + 4) + 8 * d)) + 4 * pages, "flops": 3 * keys * kv * d}
    h, row = case["heads"], _row_bytes(case)
    if op == "select":
        scored = [(t - 1) // p + 1 for t in total]
        pairs = sum((t - a + j) // p + 1 for a, t in zip(new, total) for j in range(a))
        return {"bytes": sum(scored) * kv * (2 * d + 4) + sum(new) * (h * row + 4 * kv * case["n_select"]), "flops": pairs * kv * 4 * d + 2 * sum(new) * h * d}
    # a request's pages count once, however many of its tokens read them
    reads = [[_listed_pages(t - a + j, case) for j in range(a)] for a, t in zip(new, total)]
    unique = sum(min(sum(r), -(-t // p)) for r, t in zip(reads, total))
    every = sum(sum(r) for r in reads)
    return {"bytes": 2 * sum(new) * h * row + 2 * unique * p * kv * _kv_bytes(d) + 4 * sum(new) * kv * case["n_select"], "flops": 4 * every * p * h * d}


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


def _keys_of(blocks, dim):
    """Blocks [..., block bytes]: keys [..., 16, dim] in 32 bits, before k_scale."""
    w = _width(dim)
    return _unpacked(blocks[..., : 8 * w].unflatten(-1, (16, w // 2)), blocks[..., 16 * w: 17 * w].unflatten(-1, (16, w // 16)).contiguous())[..., :dim]


def _values_of(blocks, dim):
    w = _width(dim)
    return _unpacked(blocks[..., 8 * w: 16 * w][..., _v_order(w)], blocks[..., 17 * w:].unflatten(-1, (w // 16, 16)).transpose(-1, -2).contiguous())[..., :dim]


def _random_blocks(g, m, dim):
    """m blocks of 16 tokens: rows as projections leave them, quantised with each group's largest number."""
    w = _width(dim)
    x = torch.zeros((2, m * 16, w), device=DEV)
    x[..., :dim] = _normal(g, 2, m * 16, dim) * (1.0 + 3.0 * (torch.arange(dim, device=DEV) % 29 == 5))
    scale = torch.tensor((K_SCALE, V_SCALE), device=DEV).view(2, 1, 1)
    group = x.unflatten(-1, (w // 16, 16))
    s8 = (group.abs().amax(-1) / (6.0 * scale)).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = (s8.float() * scale).unsqueeze(-1)
    y = torch.where(s > 0, group / s, torch.zeros_like(group))
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * (y < 0)).to(torch.uint8).flatten(-2)
    packed, s8 = (code[..., 0::2] | (code[..., 1::2] << 4)).unflatten(1, (m, 16)), s8.view(torch.uint8).unflatten(1, (m, 16))
    blocks = torch.zeros((m, _block_bytes(dim)), dtype=torch.uint8, device=DEV)
    blocks[:, : 8 * w] = packed[0].flatten(1)
    blocks[:, 8 * w + _v_order(w).flatten()] = packed[1].flatten(1)
    blocks[:, 16 * w: 17 * w] = s8[0].flatten(1)
    blocks[:, 17 * w:] = s8[1].transpose(1, 2).flatten(1)
    return blocks


# ---------------------------------------------------------------------------------------------- summaries, plainly

def _bounds_in_8_bits(high, low):
    """Largest and smallest numbers [..., dim] in 32 bits: (codes of both as whole numbers in 32 bits, step [..., 1])."""
    m = torch.maximum(high.abs().amax(-1, keepdim=True), low.abs().amax(-1, keepdim=True))
    some, most = torch.where(m > 0, m, torch.ones_like(m)), torch.full_like(m, 127.0)
    up, down = torch.ceil(high * 127.0 / some).clamp(-127, 127), torch.floor(low * 127.0 / some).clamp(-127, 127)
    return up, down, m / most       # a number in place of the tensor would be multiplied by its reciprocal


def _entries(high, low):
    """Summaries as they are held, [..., 2 W + 16] bytes."""
    dim, w = high.shape[-1], _width(high.shape[-1])
    up, down, step = _bounds_in_8_bits(high, low)
    out = torch.zeros(high.shape[:-1] + (2 * w + 16,), dtype=torch.uint8, device=DEV)
    out[..., :dim] = up.to(torch.int8).view(torch.uint8)
    out[..., w: w + dim] = down.to(torch.int8).view(torch.uint8)
    out[..., 2 * w: 2 * w + 4] = step.contiguous().view(torch.uint8)
    return out


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _queries(g, t, heads, dim, dtype):
    """[t, heads, dim] rows as a projection leaves them: some dimensions larger than others."""
    return (_normal(g, t, heads, dim) * (1.0 + 3.0 * (torch.arange(dim, device=DEV) % 29 == 5))).to(dtype)


def _ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _cumulative(lengths):
    return _ints([0] + lengths).cumsum(0, dtype=torch.int32)


def _cache(g, n_pages, kv, page, dim):
    """Pages whose blocks come from a store of quantised ones."""
    store = _random_blocks(g, 512, dim)
    return store[torch.randint(0, 512, (n_pages * kv * (page // 16),), generator=g, device=DEV)].view(n_pages, kv, page // 16, -1)


def _table(g, total, page, spare=3):
    """(block table of pages in any order, pages)."""
    held = _ints([-(-x // page) for x in total])
    width, n_pages = -(-max(total) // page), sum(-(-x // page) for x in total) + spare
    table = torch.full((len(total), width), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV) < held.view(-1, 1)] = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int32)[: n_pages - spare]
    return table, n_pages


def _plan(case, requests, tokens):
    from paper_2509_02753_b200 import kv_cache
    return kv_cache.KVPlan(n_heads=case.get("heads", case.get("kv_heads", 1)), n_kv_heads=case.get("kv_heads", 1), head_dim=case.get("head_dim", 64), page_size=case["page"],
                           dtype=_TYPES[case.get("dtype", "bf16")], max_requests=requests, max_tokens=tokens)


def prepare(case, seed):
    g, op, p = _gen(seed), case["op"], case["page"]
    if op in ("prefix", "shared"):
        cu, pages, new, total = _groups(case)
        table, n_pages = _table(g, total, p)
        for j, m in enumerate(pages):         # the first member's pages are all members'; where the length is to be found, up to half of them is not
            common = m - (torch.rand((), generator=g, device=DEV) * torch.rand((cu[j + 1] - cu[j], 1), generator=g, device=DEV) * (m / 2 + 1)).int() if op == "prefix" else m
            member = table[cu[j]: cu[j + 1]]
            member.copy_(torch.where(torch.arange(table.shape[1], device=DEV) < common, table[cu[j]].clone(), member))
        state = {"groups": _ints(cu)}
        if op == "shared":
            state |= {"shared": _ints([m * p if cu[j + 1] - cu[j] > 1 else 0 for j, m in enumerate(pages)]), "cu_group": cu, "pages": pages, "max_group": max(b - a for a, b in zip(cu, cu[1:])) * case["new"],
                      "start": torch.cat([_ints([m * p if cu[j + 1] - cu[j] > 1 else 0]).expand(cu[j + 1] - cu[j]) for j, m in enumerate(pages)])}
            # no holes: the cache has the pages that are in use
            used, table_of = torch.unique(table.clamp(min=0), return_inverse=True)
            table, n_pages = torch.where(table >= 0, table_of.int(), table), used.numel()
    else:
        new, total = _lengths(case)
        table, n_pages = _table(g, total, p)
        state = {}
    state |= {"case": case, "cu": _cumulative(new), "len": _ints(total), "table": table, "tokens": sum(new), "max_new": max(new), "longest": max(total)}
    if op in ("shared", "summarise", "selected"):
        state["cache"] = _cache(g, n_pages, case["kv_heads"], p, case["head_dim"])
    if op == "summarise":
        at = [(i, c) for i, (a, t) in enumerate(zip(new, total)) for c in range((t - a) // p, -(-t // p))]
        state["where"] = torch.tensor(at, device=DEV).t().contiguous()
        state["pages"] = table[state["where"][0], state["where"][1]]
        state["summaries"] = torch.zeros((n_pages, case["kv_heads"], 2 * _width(case["head_dim"]) + 16), dtype=torch.uint8, device=DEV)
    if op in ("shared", "select", "selected"):
        state["q"] = _queries(g, sum(new), case["heads"], case["head_dim"], _TYPES[case["dtype"]])
    if op == "select":
        kv, d = case["kv_heads"], case["head_dim"]
        middle, reach = _normal(g, n_pages, kv, d), 1.0 + _normal(g, n_pages, kv, d).abs()
        loud = 30.0 * (1.0 + 3.0 * (torch.arange(d, device=DEV) % 29 == 5))
        state["summaries"] = _entries((middle + reach) * loud, (middle - reach) * loud)
    if op == "selected":
        # as a selection leaves them: ascending, the first and the last pages among them, -1 behind
        t, kv, m = sum(new), case["kv_heads"], case["n_select"]
        request = torch.repeat_interleave(torch.arange(len(new), device=DEV), torch.tensor(new, device=DEV))
        at = state["len"][request].long() - torch.tensor(new, device=DEV)[request] + torch.arange(t, device=DEV) - state["cu"][request].long()
        own_page = (at // p).view(-1, 1, 1)
        col = torch.arange(max(table.shape[1], m), device=DEV)
        rank = torch.rand((t, kv, col.numel()), generator=g, device=DEV)
        rank = torch.where((col < case["first"]) | (col > own_page - case["last"]), torch.full_like(rank, 2.0), rank)
        rank = torch.where(col <= own_page, rank, torch.full_like(rank, -1.0))
        value, index = rank.topk(m, -1)
        index = torch.where(value >= 0, index, torch.full_like(index, 1 << 30)).sort(-1).values
        state["selected"] = torch.where(index < (1 << 30), index, torch.full_like(index, -1)).int()
    if own:
        state["plan"] = _plan(case, case["requests"], max(1, sum(new)))
    return state


# ---------------------------------------------------------------------------------------------- the operators, plainly

def _prefix(groups, cu, lens, table, page):
    n, width = table.shape
    g = groups.numel() - 1
    new = cu[1:] - cu[:-1]
    full = torch.div(lens - new, page, rounding_mode="floor")
    member = torch.searchsorted(groups[1:].contiguous(), torch.arange(n, device=DEV, dtype=torch.int32), right=True)
    lead = table[groups[:-1].long()[member]]
    col = torch.arange(width, device=DEV)
    same = (table == lead) & (table >= 0) & (col < full.view(-1, 1))
    leading = same.int().cumprod(1).sum(1).int()
    pages = torch.full((g,), width, dtype=torch.int32, device=DEV).scatter_reduce(0, member, leading, "amin")
    shared = torch.where(groups[1:] - groups[:-1] > 1, pages * page, torch.zeros_like(pages))
    return shared, shared[member]


def _softmaxed(parts):
    """[(scores [..., rows, keys], values [..., keys, dim])]: the softmax over all of them together, [..., rows, dim]."""
    top = torch.stack([s.amax(-1, keepdim=True) for s, _ in parts]).amax(0)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    total, out = 0.0, 0.0
    for s, v in parts:
        w = s.sub_(top).exp_()
        total = total + w.sum(-1, keepdim=True)
        out = out + torch.matmul(w, v)
    return out.mul_(V_SCALE) / torch.where(total > 0, total, torch.ones_like(total))


def _shared(state, case):
    q, table, cache, lens, p, d, kv, a = (state["q"], state["table"], state["cache"], state["len"], case["page"], case["head_dim"], case["kv_heads"], case["new"])
    h = case["heads"]
    g = h // kv
    scale = K_SCALE / math.sqrt(d)
    out = torch.empty_like(q)
    for j, pages in enumerate(state["pages"]):
        lo, hi = state["cu_group"][j], state["cu_group"][j + 1]
        m = hi - lo
        rows = q[lo * a: hi * a].float().view(m, a, kv, g, d)
        blocks = cache[table[lo, :pages].long()].transpose(0, 1).flatten(1, 2)            # [kv, blocks, bytes]
        k, v = _keys_of(blocks, d).flatten(1, 2), _values_of(blocks, d).flatten(1, 2)
        every = rows.permute(2, 0, 1, 3, 4).reshape(kv, m * a * g, d)
        parts = []
        if pages:
            parts.append((torch.matmul(every, k.transpose(-1, -2)).mul_(scale).view(kv, m, a * g, -1), v.unsqueeze(1)))
        blocks = cache[table[lo:hi, pages:].clamp(min=0).long()].permute(2, 0, 1, 3, 4).flatten(2, 3)      # [kv, m, blocks, bytes]
        k, v = _keys_of(blocks, d).flatten(2, 3), _values_of(blocks, d).flatten(2, 3)
        s = torch.matmul(every.view(kv, m, a * g, d), k.transpose(-1, -2)).mul_(scale).view(kv, m, a, g, -1)
        key = pages * p + torch.arange(s.shape[-1], device=DEV)
        at = (lens[lo:hi] - a).view(-1, 1) + torch.arange(a, device=DEV)
        s.masked_fill_(key > at.view(1, m, a, 1, 1), -math.inf)
        parts.append((s.flatten(2, 3), v))
        o = _softmaxed(parts)
        out[lo * a: hi * a] = o.view(kv, m, a, g, d).permute(1, 2, 0, 3, 4).reshape(m * a, h, d).to(q.dtype)
    return out


def _summarised(state, case):
    request, col = state["where"]
    d, p = case["head_dim"], case["page"]
    k = _keys_of(state["cache"][state["pages"].long()], d).flatten(2, 3)             # [m, kv, page, dim]
    held = (torch.arange(p, device=DEV) < (state["len"][request] - col * p).view(-1, 1)).view(-1, 1, p, 1)
    high, low = k.masked_fill(~held, -math.inf).amax(2), k.masked_fill(~held, math.inf).amin(2)
    up, down, step = _bounds_in_8_bits(high, low)
    return up * step * K_SCALE, down * step * K_SCALE


def _in_8_bits(x):
    """Rows of numbers in 32 bits as whole numbers up to 127."""
    m = x.abs().amax(-1, keepdim=True)
    return torch.round(x * (torch.full_like(m, 127.0) / torch.where(m > 0, m, torch.ones_like(m))))


def _select(q, cu, lens, table, summaries, longest, max_new, case):
    t, h, d = q.shape
    n, kv, w, p, m, first, last = lens.numel(), case["kv_heads"], _width(case["head_dim"]), case["page"], case["n_select"], case["first"], case["last"]
    pages = (longest - 1) // p + 1
    high_q = torch.zeros((t, kv, d), device=DEV)
    low_q = torch.zeros((t, kv, d), device=DEV)
    rows = q.float().view(t, kv, h // kv, d)
    for i in range(h // kv):                # sums in the order of the heads
        high_q = high_q + rows[:, :, i].clamp(min=0)
        low_q = low_q + rows[:, :, i].clamp(max=0)
    rows = _in_8_bits(torch.cat((high_q, low_q), -1))
    new = (cu[1:] - cu[:-1]).view(-1, 1)
    row = torch.arange(max_new, device=DEV).view(1, -1)
    real = row < new
    source = (cu[:-1].view(-1, 1) + row).clamp(max=t - 1).long()
    entry = summaries[table[:, :pages].clamp(min=0).long()]                  # [n, pages, kv, bytes]
    bounds = torch.cat((entry[..., :d], entry[..., w: w + d]), -1).view(torch.int8).float()
    step = entry[..., 2 * w: 2 * w + 4].contiguous().view(torch.float32)[..., 0]
    # whole numbers below 2^24, whatever the order of the sum
    s = torch.matmul(rows[source].transpose(1, 2), bounds.permute(0, 2, 3, 1)) * step.permute(0, 2, 1).unsqueeze(2)      # [n, kv, max_new, pages]
    own_page = torch.div(lens.view(-1, 1) - new + row, p, rounding_mode="floor").view(n, 1, max_new, 1)
    col = torch.arange(pages, device=DEV)
    s = torch.where((col < first) | (col > own_page - last), torch.full_like(s, math.inf), s)
    s = torch.where(col <= own_page, s, torch.full_like(s, -math.inf))
    order = s.sort(dim=-1, descending=True, stable=True)
    index = torch.where(order.values > -math.inf, order.indices, torch.full_like(order.indices, 1 << 30))[..., :m].sort(-1).values
    index = torch.nn.functional.pad(index, (0, max(0, m - pages)), value=1 << 30)
    index = torch.where(index < (1 << 30), index, torch.full_like(index, -1)).int()
    return index.permute(0, 2, 1, 3)[real]


def _selected(q, cu, lens, table, cache, selected, case):
    t, h, d = q.shape
    kv, p, m = case["kv_heads"], case["page"], case["n_select"]
    out = torch.empty_like(q)
    request = torch.searchsorted(cu[1:].contiguous(), torch.arange(t, device=DEV, dtype=torch.int32), right=True)
    at = lens[request] - (cu[1:] - cu[:-1])[request] + torch.arange(t, device=DEV, dtype=torch.int32) - cu[request]
    few = max(1, (1 << 26) // (kv * m * p * _width(d)))
    for lo in range(0, t, few):              # the keys of a few tokens at a time
        pick, r = selected[lo: lo + few], request[lo: lo + few]
        page = table[r.view(-1, 1, 1), pick.clamp(min=0).long()].clamp(min=0).long()
        blocks = cache[page, torch.arange(kv, device=DEV).view(1, -1, 1)].flatten(2, 3)             # [few, kv, blocks, bytes]
        k, v = _keys_of(blocks, d).flatten(2, 3), _values_of(blocks, d).flatten(2, 3)
        s = torch.matmul(q[lo: lo + few].float().view(-1, kv, h // kv, d), k.transpose(-1, -2)).mul_(K_SCALE / math.sqrt(d))
        key = (pick.unsqueeze(-1) * p + torch.arange(p, device=DEV)).flatten(2)
        see = (key >= 0) & (key <= at[lo: lo + few].view(-1, 1, 1))
        s.masked_fill_(~see.unsqueeze(2), -math.inf)
        out[lo: lo + few] = _softmaxed([(s, v)]).reshape(-1, h, d).to(q.dtype)
    return out


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        return _run_own(state, case, op)
    if op == "prefix":
        shared, start = _prefix(state["groups"], state["cu"], state["len"], state["table"], case["page"])
        return {"shared": shared, "start": start}
    if op == "shared":
        return _shared(state, case)
    if op == "summarise":
        high, low = _summarised(state, case)
        return {"high": high, "low": low}
    if op == "select":
        return _select(state["q"], state["cu"], state["len"], state["table"], state["summaries"], state["longest"], state["max_new"], case)
    return _selected(state["q"], state["cu"], state["len"], state["table"], state["cache"], state["selected"], case)


def _run_own(state, case, op):
    plan = state["plan"]
    if op == "prefix":
        shared, start = plan.shared_prefix(state["groups"], state["cu"], state["len"], state["table"])
        return {"shared": shared, "start": start}
    if op == "shared":
        return plan.attention_shared(state["q"], state["cu"], state["len"], state["table"], state["cache"], state["groups"], state["shared"], state["start"],
                                     max_new=state["max_new"], max_group=state["max_group"], k_scale=K_SCALE, v_scale=V_SCALE)
    if op == "summarise":
        plan.summarise(state["cu"], state["len"], state["table"], state["cache"], state["summaries"], state["tokens"])
        high, low = plan.read_summaries(state["summaries"], state["pages"], k_scale=K_SCALE)
        return {"high": high, "low": low}
    if op == "select":
        return plan.select(state["q"], state["cu"], state["len"], state["table"], state["summaries"], n_select=case["n_select"], first=case["first"], last=case["last"],
                           max_new=state["max_new"])
    return plan.attention_selected(state["q"], state["cu"], state["len"], state["table"], state["cache"], state["selected"], k_scale=K_SCALE, v_scale=V_SCALE)


# ---------------------------------------------------------------------------------------------- the operators' definitions in 64 bits

def _exact_blocks(block, dim):
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


def _exact_attention(q, k, v, see):
    """q [t, heads, dim], k and v [keys, dim], see [t, keys] or none: [t, heads, dim] in 64 bits."""
    s = torch.einsum("tgd,kd->gtk", q.double(), k * K_SCALE) / math.sqrt(q.shape[-1])
    if see is not None:
        s = s.masked_fill(~see, -math.inf)
    return torch.einsum("gtk,kd->tgd", torch.softmax(s, -1), v * V_SCALE)


def exact(case, seed):
    op, p = case["op"], case["page"]
    if op in ("prefix", "select"):
        return None
    state = prepare(case, seed)
    d, kv = case["head_dim"], case["kv_heads"]
    if op == "summarise":
        high, low = [], []
        for (i, c), page in zip(state["where"].t().tolist(), state["pages"].tolist()):
            held = min(p, int(state["len"][i]) - c * p)
            k = torch.stack([_exact_blocks(state["cache"][page, j], d)[0].reshape(-1, d)[:held] for j in range(kv)])
            most, least = k.amax(1), k.amin(1)
            m = torch.maximum(most.abs(), least.abs()).amax(-1, keepdim=True)
            step = m / 127
            some = torch.where(m > 0, m, torch.ones_like(m))
            high.append(torch.ceil(most * 127 / some) * step * K_SCALE)
            low.append(torch.floor(least * 127 / some) * step * K_SCALE)
        return {"high": torch.stack(high), "low": torch.stack(low)}
    h = case["heads"]
    g = h // kv
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device=DEV)
    if op == "shared":
        if 2.0 * work(case)["flops"] > 3e12:
            return None
        _, _, new, total = _groups(case)
        at = 0
        for i, (a, m) in enumerate(zip(new, total)):
            pages = state["table"][i, : -(-m // p)].long()
            see = torch.arange(m, device=DEV) <= torch.arange(m - a, m, device=DEV).view(-1, 1)
            for j in range(kv):
                k, v = (x.reshape(-1, d)[:m] for x in _exact_blocks(state["cache"][pages, j].flatten(0, 1), d))
                out[at: at + a, j * g: (j + 1) * g] = _exact_attention(state["q"][at: at + a, j * g: (j + 1) * g], k, v, see)
            at += a
        return out
    new, total = _lengths(case)
    if sum(new) * kv > 4000:
        return None
    t = 0
    for i, (a, m) in enumerate(zip(new, total)):
        for row in range(m - a, m):
            for j in range(kv):
                pick = state["selected"][t, j]
                pick = pick[pick >= 0].long()
                k, v = (x.reshape(-1, d) for x in _exact_blocks(state["cache"][state["table"][i, pick].long(), j].flatten(0, 1), d))
                key = (pick.view(-1, 1) * p + torch.arange(p, device=DEV)).flatten()
                out[t: t + 1, j * g: (j + 1) * g] = _exact_attention(state["q"][t: t + 1, j * g: (j + 1) * g], k, v, (key <= row).view(1, -1))
            t += 1
    return out
