"""The definitions of the cache in 4 bits and of the verification of drafted tokens, in 64 bits (numpy).  Nothing here touches the library."""
import numpy as np

import layer_plain as plain


def half(x):
    """to fp16 by way of fp32"""
    with np.errstate(over="ignore"):
        return np.asarray(x, np.float64).astype(np.float32).astype(np.float16)


def sizes(dim, group):
    return 16 * -(-dim // 32), -(-dim // group)


def page_bytes(kv_heads, dim, page, group):
    row, groups = sizes(dim, group)
    return kv_heads * page * (row + 4 * groups)


def quantise(x, group):
    """codes (-8 .. 7) [..][dim], scales and middles fp16 [..][groups] of x [..][dim]"""
    x = np.asarray(x, np.float64)
    dim, n = x.shape[-1], -(-x.shape[-1] // group)
    codes = np.zeros(x.shape, np.int64)
    scales, middles = (np.zeros(x.shape[:-1] + (n,), np.float16) for _ in range(2))
    for g in range(n):
        y = x[..., g * group:min(dim, (g + 1) * group)]
        fine = np.isfinite(y).all(axis=-1)
        y = np.clip(np.where(np.isfinite(y), y, 0), -32768, 32768)
        lo, hi = y.min(axis=-1), y.max(axis=-1)
        scale = half((hi - lo) / 15)
        middle = half(lo + 8 * scale.astype(np.float64))
        s, m = (v.astype(np.float64)[..., None] for v in (scale, middle))
        c = np.clip(np.rint((y - m) / np.where(s > 0, s, 1)), -8, 7)
        codes[..., g * group:min(dim, (g + 1) * group)] = np.where(fine[..., None] & (s > 0), c, 0)
        scales[..., g], middles[..., g] = np.where(fine, scale, np.float16(np.nan)), np.where(fine, middle, np.float16(0))
    return codes, scales, middles


def pack(x, group):
    """rows of codes [..][row bytes] and of pairs [..][groups][2] of x [..][dim], as they lie in a page"""
    codes, scales, middles = quantise(x, group)
    row, _ = sizes(x.shape[-1], group)
    nibbles = np.zeros(x.shape[:-1] + (2 * row,), np.uint8)
    nibbles[..., :x.shape[-1]] = codes + 8
    pairs = np.stack([scales, middles], axis=-1)
    bits = pairs.view(np.uint16)
    bits[np.isnan(pairs)] = 0x7E00
    return nibbles[..., 0::2] | nibbles[..., 1::2] << 4, pairs


def values(codes, pairs, dim, group):
    """what rows of codes and pairs stand for, [..][dim]"""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[:-1] + (-1,))[..., :dim].astype(np.float64) - 8
    f = np.arange(dim) // group
    with np.errstate(invalid="ignore", over="ignore"):
        return (pairs[..., f, 1].astype(np.float64) + pairs[..., f, 0].astype(np.float64) * c).astype(np.float16).astype(np.float64)


def parts(pool, kv_heads, dim, page, group):
    """codes [page][head][slot][bytes] and pairs [page][head][slot][groups][2] of a pool [page][bytes], as views"""
    row, groups = sizes(dim, group)
    x = pool.reshape(pool.shape[0], kv_heads, -1)
    return x[:, :, :page * row].reshape(-1, kv_heads, page, row), x[:, :, page * row:].view(np.float16).reshape(-1, kv_heads, page, groups, 2)


def pool_of(x, group, fill=0xFF):
    """A pool's bytes for values x [page][head][slot][dim]; rows that are NaN throughout are places that nothing was written to, and hold `fill`."""
    n, heads, page, dim = x.shape
    row, groups = sizes(dim, group)
    codes, pairs = pack(x, group)
    empty = np.isnan(x).all(axis=-1)
    codes[empty] = fill
    pairs.view(np.uint16)[empty] = fill | fill << 8
    return np.concatenate([codes.reshape(n, heads, -1), pairs.reshape(n, heads, -1).view(np.uint8).reshape(n, heads, -1)], axis=2).reshape(n, -1).copy()


def rotated(x, cos, sin, style):
    """in 64 bits; x [dim], cos and sin fp32 rows"""
    return plain.rotate(np.asarray(x, np.float64), np.asarray(cos, np.float64), np.asarray(sin, np.float64), style)


def append(codes_K, pairs_K, codes_V, pairs_V, c, cos, sin, style, group):
    """The step of a layer_plain.Case into parts() of both pools, in place"""
    for b in range(len(c.cu) - 1):
        for i in range(c.cu[b + 1] - c.cu[b]):
            t, slot = c.cu[b] + i, max(c.lens[b], 0) + i
            if slot >= c.max_len:
                continue
            pos = c.prefix + slot
            k = rotated(c.k[t], cos[pos], sin[pos], style) if cos is not None else c.k[t]
            page, at = plain.place(c.pages[b], c.page, slot)
            codes_K[page, :, at], pairs_K[page, :, at] = pack(k, group)
            codes_V[page, :, at], pairs_V[page, :, at] = pack(np.asarray(c.v[t], np.float64), group)


def verify(p, q, drafted, cu, u, r):
    """tokens, accepted"""
    tokens, accepted = np.full(len(drafted), -1, np.int32), np.zeros(len(cu) - 1, np.int32)
    vocab = p.shape[1]
    for b, (lo, hi) in enumerate(zip(cu, cu[1:])):
        if lo == hi:
            continue
        row = lo
        while row < hi - 1:
            d = drafted[row]
            if not (0 <= d < vocab) or not np.float32(u[row]) * (np.float32(1) if q is None else q[row, d]) < p[row, d]:
                break
            tokens[row] = d
            row += 1
        w = p[row].copy()
        if row < hi - 1 and 0 <= drafted[row] < vocab:
            if q is None:
                w[drafted[row]] = 0
            else:
                w = np.maximum(p[row] - q[row], np.float32(0))
        if not w.max() > 0:
            w = p[row]
        run = np.cumsum(w.astype(np.float64))
        tokens[row] = min(int(np.searchsorted(run, float(r[b]) * run[-1], side="right")), vocab - 1)
        accepted[b] = row - lo
    return tokens, accepted
