"""The definitions of the operators around the FF block, in 64 bits (numpy), and inputs for them.  Nothing here touches the library."""
import numpy as np

import synth


def stored(a, dtype):
    """values as the storage type holds them, as float64"""
    return synth.store(np.asarray(a, np.float32), dtype).astype(np.float64)


# ----------------------------------------------------------------------------------------------- norms
def unit(v, w, b, *, layer, eps, offset):
    if layer:
        v = v - v.mean(axis=-1, keepdims=True)
    out = v / np.sqrt((v * v).mean(axis=-1, keepdims=True) + eps) * (w + offset)
    return out if b is None else out + b


def norm_residual(h, y, gate, w_pre, b_pre, w_post, b_post, *, layer, eps, offset, h_scale, y_scale):
    if y is not None:
        u = y if w_post is None else unit(y, w_post, b_post, layer=layer, eps=eps, offset=offset)
        h = h_scale * h + y_scale * (u if gate is None else gate * u)
    return h, None if w_pre is None else unit(h, w_pre, b_pre, layer=layer, eps=eps, offset=offset)


# ----------------------------------------------------------------------------------------------- the cache
def rotate(x, cos, sin, style):
    """x [..., dim] with cos, sin [..., rot / 2] that broadcast against it"""
    half = cos.shape[-1]
    out = np.array(x, dtype=np.float64)
    a, b = (slice(0, half), slice(half, 2 * half)) if style == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    out[..., a] = x[..., a] * cos - x[..., b] * sin
    out[..., b] = x[..., b] * cos + x[..., a] * sin
    return out


def place(pages, page_size, slot):
    return pages[slot // page_size], slot % page_size


def append(K, V, k, v, q, cos, sin, style, cu, lens, pages, page_size, n_prefix, max_len):
    """K, V [page][head][slot][dim] in place; returns the rotated queries"""
    q_out = np.array(q)
    for b in range(len(cu) - 1):
        for i in range(cu[b + 1] - cu[b]):
            t, slot = cu[b] + i, max(lens[b], 0) + i
            pos = n_prefix + slot
            c, s = (cos[pos], sin[pos]) if cos is not None else (np.zeros(0), np.zeros(0))
            q_out[t] = rotate(q[t], c, s, style)
            if slot < max_len:
                page, at = place(pages[b], page_size, slot)
                K[page, :, at], V[page, :, at] = rotate(k[t], c, s, style), v[t]
    return q_out


# ----------------------------------------------------------------------------------------------- attention
def attention(q, K, V, cu, lens, pages, prefix_pages, page_size, n_prefix, max_len, scale):
    """out and, beside it, sum p |v|: what an error of the weights can do"""
    T, heads, dim = q.shape
    kvh = K.shape[1]
    group = heads // kvh
    out, size = np.zeros((T, heads, dim)), np.zeros((T, heads, dim))
    shared = [place(prefix_pages, page_size, i) for i in range(n_prefix)]
    for b in range(len(cu) - 1):
        n, held = cu[b + 1] - cu[b], max(lens[b], 0)
        if n == 0:
            continue
        where = shared + [place(pages[b], page_size, i) for i in range(min(held + n, max_len))]
        page, at = (np.array(x) for x in zip(*where))
        for i in range(n):
            see = n_prefix + min(held + i + 1, max_len)
            for h in range(kvh):
                k, v = K[page[:see], h, at[:see]], V[page[:see], h, at[:see]]
                s = q[cu[b] + i, h * group:(h + 1) * group] @ k.T * scale
                p = np.exp(s - s.max(axis=-1, keepdims=True))
                p /= p.sum(axis=-1, keepdims=True)
                with np.errstate(invalid="ignore"):
                    out[cu[b] + i, h * group:(h + 1) * group] = p @ v
                    size[cu[b] + i, h * group:(h + 1) * group] = p @ np.abs(v)
    return out, size


class Case:
    """Pools, page tables and new tokens of one step.  What no token may see is NaN: pages that nobody has, slots behind a sequence's
    last token."""

    def __init__(self, seed, *, heads, kv_heads, dim, page, prefix, held, new, dtype, max_len=None, q_scale=1.0):
        rng = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.dim, self.page, self.prefix, self.dtype = heads, kv_heads, dim, page, prefix, dtype
        self.lens, self.new = list(held), list(new)
        self.cu = [0] + [int(x) for x in np.cumsum(new)]
        self.max_len = max_len or max(1, max(max(h, 0) + n for h, n in zip(held, new)))
        up = lambda n: -(-n // page)  # noqa: E731
        width = up(self.max_len)
        own = [up(min(max(h, 0) + n, self.max_len)) for h, n in zip(held, new)]
        self.n_pages = up(prefix) + sum(own) + 3
        order = rng.permutation(self.n_pages)
        self.prefix_pages = order[:up(prefix)].astype(np.int32)
        self.pages = np.full((len(new), width), order[-1], dtype=np.int32)       # entries that are not in use name a page of NaN
        at = up(prefix)
        for b, c in enumerate(own):
            self.pages[b, :c] = order[at:at + c]
            at += c
        shape = (self.n_pages, kv_heads, page, dim)
        self.K, self.V = (stored(rng.standard_normal(shape), dtype) for _ in range(2))
        used = np.zeros((self.n_pages, page), bool)
        for i in range(prefix):
            used[place(self.prefix_pages, page, i)] = True
        for b in range(len(new)):
            for i in range(min(max(held[b], 0) + new[b], self.max_len)):
                used[place(self.pages[b], page, i)] = True
        for pool in (self.K, self.V):
            pool[~used[:, None, :].repeat(kv_heads, axis=1)] = np.nan
        T = self.cu[-1]
        self.q = stored(rng.standard_normal((T, heads, dim)) * q_scale, dtype)
        self.k, self.v = (stored(rng.standard_normal((T, kv_heads, dim)), dtype) for _ in range(2))

    def attention(self, scale):
        return attention(self.q, self.K, self.V, self.cu, self.lens, self.pages, self.prefix_pages, self.page, self.prefix, self.max_len, scale)
