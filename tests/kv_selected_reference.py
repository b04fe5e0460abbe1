"""Plain implementations of the operators around shared prefixes and selected pages for the tests: numpy, loops; 32 bits
operation by operation where whole numbers come of it (what is selected has to be equal), 64 bits where numbers are computed."""
import numpy as np

import kv_reference as ref

F = np.float32


def decode_all(cache, dim):
    """kv_reference.decode_all, all bytes at once."""
    w = ref.width(dim)
    token, d = np.arange(16)[:, None], np.arange(dim)[None, :]
    shift = 4 * (d % 2) + 0 * token
    parts = ((token * (w // 2) + d // 2, 16 * w + token * (w // 16) + d // 16), (ref.value_at(w, token, d)[0], 17 * w + d // 16 * 16 + token))
    scale = ref.e4m3_value(np.arange(256))
    code = np.concatenate((ref.GRID, -ref.GRID))
    out = []
    for at, sc in parts:
        x = code[(cache[..., at] >> shift) & 15] * scale[cache[..., sc]]
        out.append(x.reshape(*cache.shape[:2], -1, dim))
    return out


def store(cache, k, v, slots, page, k_scale, v_scale):
    """kv_reference.store, all rows at once; no slot twice."""
    dim, slots = k.shape[-1], np.asarray(slots)
    w = ref.width(dim)
    token, d, g = (slots % 16)[:, None, None], np.arange(0, w, 2)[None, None, :], np.arange(w // 16)[None, None, :]
    where = (slots // page)[:, None, None], np.arange(k.shape[1])[None, :, None], (slots % page // 16)[:, None, None]
    for x, factor, key in ((k, k_scale, True), (v, v_scale, False)):
        codes, scales = ref.quantise(x, factor)
        at = token * (w // 2) + d // 2 if key else ref.value_at(w, token, d)[0]
        cache[where + (at,)] = codes[..., 0::2] | (codes[..., 1::2] << 4)
        cache[where + (16 * w + token * (w // 16) + g if key else 17 * w + g * 16 + token,)] = scales


def shared_prefix(groups, cu, kv_len, table, page):
    n, width = table.shape
    shared, start = [], [0] * n
    for g in range(len(groups) - 1):
        members = range(groups[g], groups[g + 1])
        pages = 0
        if len(members) > 1:
            most = min([width] + [max(int(kv_len[i]) - (cu[i + 1] - cu[i]), 0) // page for i in members])
            while pages < most and all(table[i, pages] == table[members[0], pages] >= 0 for i in members):
                pages += 1
        shared.append(pages * page)
        for i in members:
            start[i] = pages * page
    return shared, start


def summary(keys):
    """keys [tokens, dim] in 64 bits, before k_scale: (codes of the largest, of the smallest, step)."""
    high, low = keys.max(0), keys.min(0)
    m = max(np.abs(high).max(), np.abs(low).max())
    if m == 0:
        return np.zeros(len(high), int), np.zeros(len(high), int), F(0)
    return np.ceil(high * 127 / m).astype(int), np.floor(low * 127 / m).astype(int), F(m / 127)


def entry(codes_high, codes_low, step, dim):
    """The bytes that are held."""
    w = ref.width(dim)
    out = np.zeros(2 * w + 16, np.uint8)
    out[:dim] = codes_high.astype(np.int8).view(np.uint8)
    out[w: w + dim] = codes_low.astype(np.int8).view(np.uint8)
    out[2 * w: 2 * w + 4] = np.array([step], F).view(np.uint8)
    return out


def in_8_bits(u, w):
    """Both vectors as whole numbers, the largest magnitude at 127."""
    m = max(u.max(), (-w).max())
    if not m > 0:
        return np.zeros(len(u), np.int64), np.zeros(len(w), np.int64)
    with np.errstate(over="ignore", invalid="ignore"):
        inv = F(127) / F(m)
        a, b = np.rint((u * inv).astype(F)), np.rint((w * inv).astype(F))
    return tuple(np.clip(np.nan_to_num(x, nan=0.0, posinf=127, neginf=-127), -127, 127).astype(np.int64) for x in (a, b))


def select(q, cu, kv_len, table, summaries, heads, page, n_select, first, last):
    """q [T, H, dim] as fp32 numbers; summaries [pages, heads, bytes]; rows of tokens of no request are -2."""
    T, H, dim = q.shape
    G, w = H // heads, ref.width(dim)
    out = np.full((T, heads, n_select), -2)
    for i in range(len(kv_len)):
        for t in range(cu[i], cu[i + 1]):
            p = int(kv_len[i]) - (cu[i + 1] - t)
            own = p // page if p >= 0 else -1
            for h in range(heads):
                out[t, h] = -1
                if own < n_select:
                    out[t, h, : own + 1] = np.arange(own + 1)
                    continue
                u, v = np.zeros(dim, F), np.zeros(dim, F)
                for g in range(G):
                    x = np.nan_to_num(q[t, h * G + g], nan=0.0, posinf=np.inf, neginf=-np.inf).astype(F)
                    u, v = u + np.maximum(x, F(0)), v + np.minimum(x, F(0))
                a, b = in_8_bits(u, v)
                scored = []
                for c in range(first, own - last + 1):
                    pg = int(table[i, c])
                    e = summaries[pg, h] if 0 <= pg < len(summaries) else np.zeros(2 * w + 16, np.uint8)
                    whole = int(e[:dim].view(np.int8).astype(np.int64) @ a + e[w: w + dim].view(np.int8).astype(np.int64) @ b)
                    scored.append((-(F(whole) * e[2 * w: 2 * w + 4].view(F)[0]), c))
                best = sorted(c for _, c in sorted(scored)[: n_select - first - last])
                out[t, h] = list(range(first)) + best + list(range(own - last + 1, own + 1))
    return out


def attention_selected(q, cu, kv_len, table, cache, selected, page, scale, k_scale, v_scale):
    """(out, spread, exponent, count) as kv_reference.attention; columns outside the table count as none."""
    T, H, dim = q.shape
    heads = cache.shape[1]
    G = H // heads
    k_all, v_all = decode_all(cache, dim)
    out, spread, exponent, count = np.zeros((T, H, dim)), np.zeros((T, H, dim)), np.zeros((T, H, 1)), np.ones((T, H, 1))
    for i in range(len(kv_len)):
        for t in range(cu[i], cu[i + 1]):
            p = int(kv_len[i]) - (cu[i + 1] - t)
            for h in range(heads):
                at = [(int(table[i, c]), j) for c in selected[t, h] if 0 <= c < table.shape[1] for j in range(page) if c * page + j <= p]
                at = [(pg, j) for pg, j in at if 0 <= pg < len(cache)]
                if not at:
                    continue
                pg, j = (np.array(x) for x in zip(*at))
                k, v = k_all[pg, h, j] * k_scale, v_all[pg, h, j] * v_scale
                for g in range(G):
                    row = q[t, h * G + g].astype(np.float64)
                    x = (k @ row) * scale
                    weight = np.exp(x - x.max())
                    weight /= weight.sum()
                    r = (t, h * G + g)
                    out[r], spread[r] = weight @ v, weight @ np.abs(v)
                    exponent[r] = (np.abs(k) @ np.abs(row)).max() * abs(scale)
                    count[r] = len(at)
    return out, spread, exponent, count


def attention(q, cu, kv_len, table, cache, page, scale, k_scale, v_scale):
    """(out, spread, exponent, count) as kv_reference.attention without a window, a request's rows at once; every page is in the cache."""
    T, H, dim = q.shape
    heads = cache.shape[1]
    G = H // heads
    out, spread, exponent, count = np.zeros((T, H, dim)), np.zeros((T, H, dim)), np.zeros((T, H, 1)), np.ones((T, H, 1))
    for i in range(len(kv_len)):
        n, rows = int(kv_len[i]), slice(cu[i], cu[i + 1])
        new = cu[i + 1] - cu[i]
        if n == 0 or new == 0:
            continue
        k, v = (x.transpose(1, 0, 2, 3).reshape(heads, -1, dim)[:, :n] * s for x, s in zip(decode_all(cache[table[i, : -(-n // page)]], dim), (k_scale, v_scale)))
        row = q[rows].astype(np.float64).reshape(new, heads, G, dim)
        see = np.arange(n) <= n - new + np.arange(new)[:, None]
        x = np.einsum("thgd,hkd->thgk", row, k) * scale
        x = np.where(see[:, None, None], x, -np.inf)
        top = x.max(-1, keepdims=True)
        w = np.exp(x - np.where(top > -np.inf, top, 0.0))
        w /= np.maximum(w.sum(-1, keepdims=True), 1e-300)
        out[rows] = np.einsum("thgk,hkd->thgd", w, v).reshape(new, H, dim)
        spread[rows] = np.einsum("thgk,hkd->thgd", w, np.abs(v)).reshape(new, H, dim)
        reach = np.where(see[:, None, None], np.einsum("thgd,hkd->thgk", np.abs(row), np.abs(k)), 0.0).max(-1)
        exponent[rows] = reach.reshape(new, H, 1) * abs(scale)
        count[rows] = np.maximum(see.sum(1), 1).reshape(new, 1, 1)
    return out, spread, exponent, count
