"""Plain implementations of the cache operators for the tests: numpy, loops, 64 bits where numbers are computed and 32
bits, operation by operation, where bytes are (what is stored has to be equal)."""
import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def width(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def block_bytes(dim):
    return 18 * width(dim)


def e4m3_value(byte):
    byte = np.asarray(byte).astype(np.int64)
    e, f = (byte >> 3) & 15, byte & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    return np.where((byte & 127) == 127, np.nan, v) * np.where(byte & 128, -1.0, 1.0)


_E4M3 = e4m3_value(np.arange(127))


def nearest_even(table, x):
    """Index of the entry of an increasing table nearest to x >= 0; ties to the even index; above the last: the last."""
    hi = np.clip(np.searchsorted(table, x), 1, len(table) - 1)
    lo = hi - 1
    to_lo, to_hi = x - table[lo], table[hi] - x
    up = (to_hi < to_lo) | ((to_hi == to_lo) & (hi % 2 == 0))
    return np.where(x >= table[-1], len(table) - 1, np.where(up, hi, lo))


def quantise(x, scale):
    """Rows [..., dim] fp32: (codes [..., W] 0..15, scale bytes [..., W/16])."""
    x = np.asarray(x, np.float32)
    w = width(x.shape[-1])
    x = np.nan_to_num(x, nan=0.0, posinf=np.finfo(np.float32).max, neginf=-np.finfo(np.float32).max)
    g = np.zeros(x.shape[:-1] + (w,), np.float32)
    g[..., : x.shape[-1]] = x
    g = g.reshape(x.shape[:-1] + (w // 16, 16))
    scale = np.float32(scale)
    with np.errstate(over="ignore"):
        t = np.minimum(np.abs(g).max(-1) * np.float32(1.0 / (6.0 * float(scale))), np.float32(448.0))
        byte = nearest_even(_E4M3, t.astype(np.float64))
        s = (e4m3_value(byte).astype(np.float32) * scale).astype(np.float32)
        inv = np.where(s > 0, np.float32(1.0) / np.where(s > 0, s, np.float32(1.0)), np.float32(0.0)).astype(np.float32)
        y = (g * inv[..., None]).astype(np.float32)
    code = nearest_even(GRID, np.abs(y).astype(np.float64)) + 8 * np.signbit(y)
    return code.reshape(x.shape[:-1] + (w,)).astype(np.uint8), byte.astype(np.uint8)


def value_at(w, token, d):
    """(byte, low half?) of a value code within a block."""
    r, within = d // (w // 8), d % (w // 8)
    turned = {64: 32 * ((r // 2) % 2), 128: 64 * (r % 2), 256: 16 * (r % 2)}[w]
    return 8 * w + r * w + ((token * (w // 16)) ^ turned) + within // 2, within % 2 == 0


def store(cache, k, v, slots, page, k_scale, v_scale):
    """cache [pages, heads, page/16, block bytes] uint8 numpy, in place; k, v [T, heads, dim] fp32."""
    dim = k.shape[-1]
    w = width(dim)
    for x, scale, key in ((k, k_scale, True), (v, v_scale, False)):
        codes, scales = quantise(x, scale)
        for t, slot in enumerate(slots):
            if slot < 0:
                continue
            blk = cache[slot // page, :, (slot % page) // 16]
            token = slot % 16
            for d in range(w):
                at, low = (token * (w // 2) + d // 2, d % 2 == 0) if key else value_at(w, token, d)
                old = blk[:, at]
                blk[:, at] = np.where(low, (old & 0xF0) | codes[t, :, d], (old & 0x0F) | (codes[t, :, d] << 4))
            for g in range(w // 16):
                blk[:, 16 * w + token * (w // 16) + g if key else 17 * w + g * 16 + token] = scales[t, :, g]


def load(cache, slot, page, dim):
    """Keys and values [heads, dim] in 64 bits at a slot, before k_scale and v_scale."""
    w = width(dim)
    blk = cache[slot // page, :, (slot % page) // 16].astype(np.int64)
    token = slot % 16
    k, v = np.zeros((blk.shape[0], dim)), np.zeros((blk.shape[0], dim))
    for d in range(dim):
        for out, at, low, sc in ((k, token * (w // 2) + d // 2, d % 2 == 0, 16 * w + token * (w // 16) + d // 16),
                                 (v, *value_at(w, token, d), 17 * w + d // 16 * 16 + token)):
            code = blk[:, at] & 15 if low else blk[:, at] >> 4
            out[:, d] = GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * e4m3_value(blk[:, sc])
    return k, v


def decode_all(cache, dim):
    """Every row of a cache, vectorised over pages and heads: keys and values [pages, heads, page, dim] in 64 bits."""
    w = width(dim)
    pages, heads, blocks, _ = cache.shape
    k, v = np.zeros((pages, heads, blocks, 16, dim)), np.zeros((pages, heads, blocks, 16, dim))
    b = cache.astype(np.int64)
    for token in range(16):
        for d in range(dim):
            for out, at, low, sc in ((k, token * (w // 2) + d // 2, d % 2 == 0, 16 * w + token * (w // 16) + d // 16),
                                     (v, *value_at(w, token, d), 17 * w + d // 16 * 16 + token)):
                code = b[..., at] & 15 if low else b[..., at] >> 4
                out[..., token, d] = GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * e4m3_value(b[..., sc])
    return k.reshape(pages, heads, blocks * 16, dim), v.reshape(pages, heads, blocks * 16, dim)


def rotate(x, position, turns, rot, layout, inverse=False):
    """x [T, heads, dim]; in the type of x, operation by operation."""
    y = np.array(x)
    half = rot // 2
    for t, p in enumerate(position):
        if p < 0 or p >= len(turns):
            continue
        for i in range(half):
            c, s = (x.dtype.type(z) for z in turns[p, i])
            if inverse:
                s = -s
            a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
            u, w = x[t, :, a], x[t, :, b]
            y[t, :, a] = u * c - w * s
            y[t, :, b] = w * c + u * s
    return y


def tables(ctx, new, free, table, page, capacity):
    """Loops over requests and tokens."""
    table = table.copy()
    width_ = table.shape[1]
    taken, cu, positions, slots = 0, [0], [], []
    for i, (c, m) in enumerate(zip(ctx, new)):
        c, m = max(c, 0), max(m, 0)
        held, wanted = -(-c // page), -(-(c + m) // page)
        for col in range(held, wanted):
            if col < width_:
                table[i, col] = free[taken] if taken < len(free) else -1
            taken += 1
        for j in range(m):
            p = c + j
            pg = table[i, p // page] if p // page < width_ else -1
            positions.append(p)
            slots.append(pg * page + p % page if pg >= 0 else -1)
        cu.append(cu[-1] + m)
    n = len(positions)
    positions, slots = (positions + [0] * capacity)[:capacity], (slots + [-1] * max(0, capacity - n))[:capacity]
    return table, [max(c, 0) + max(m, 0) for c, m in zip(ctx, new)], cu, positions, slots, taken


def attention(q, cu, kv_len, table, cache, page, window, sinks, scale, k_scale, v_scale):
    """(out, bound): 64 bits, loops over requests, heads and rows; bound(eps_w, terms) gives how far an output may be."""
    T, H, dim = q.shape
    heads = cache.shape[1]
    G = H // heads
    k_all, v_all = decode_all(cache, dim)
    out, spread, exponent, count = np.zeros((T, H, dim)), np.zeros((T, H, dim)), np.zeros((T, H, 1)), np.ones((T, H, 1))
    for i in range(len(kv_len)):
        n = int(kv_len[i])
        nq = cu[i + 1] - cu[i]
        pages = [int(x) for x in table[i, : -(-n // page)]]
        absent = {k for at, p in enumerate(pages) if not 0 <= p < len(cache) for k in range(at * page, (at + 1) * page)}
        pages = [p if 0 <= p < len(cache) else 0 for p in pages]
        for h in range(heads):
            k = np.concatenate([k_all[p, h] for p in pages])[:n] * k_scale if n else np.zeros((0, dim))
            v = np.concatenate([v_all[p, h] for p in pages])[:n] * v_scale if n else np.zeros((0, dim))
            for j in range(nq):
                p = n - nq + j
                keys = [x for x in range(0, p + 1) if (not window or p - x < window or x < sinks) and x not in absent]
                if not keys:
                    continue
                for g in range(G):
                    row = q[cu[i] + j, h * G + g].astype(np.float64)
                    x = (k[keys] @ row) * scale
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    at = (cu[i] + j, h * G + g)
                    out[at] = w @ v[keys]
                    spread[at] = w @ np.abs(v[keys])
                    exponent[at] = (np.abs(k[keys]) @ np.abs(row)).max() * abs(scale)
                    count[at] = len(keys)
    return out, spread, exponent, count
