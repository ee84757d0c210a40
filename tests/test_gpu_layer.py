"""What surrounds the FF block (norms and residual, paged cache, attention) against its definitions in 64 bits."""
import numpy as np
import pytest
import torch

import layer_plain as plain
import paper_2404_01365_amd as G
import synth
from devio import to_dev, to_host, workspace

pytestmark = pytest.mark.gpu

F32, BF16 = synth.DT_F32, synth.DT_BF16


def torch_type(dtype):
    return torch.bfloat16 if dtype == BF16 else torch.float32


def dev(a, dtype):
    """float64 host array with NaN and infinities in it -> device tensor; values are the storage type's own"""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch_type(dtype))


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


# ----------------------------------------------------------------------------------------------- norms
# A bf16 output is off by its own rounding (2^-8 of itself, the half of a last place of 8 significant bits).  On top, fp32: the row's sums run over at most 32 terms a lane and then a tree
# of 10 steps, so a statistic is off by some 42 x 2^-24 = 2.5e-6 at worst and half of it goes into x; a handful of products and sums
# add 2^-24 each.  Relative to the largest output of the row: 4e-6.
def norm_close(got, ref, dtype, extra=0.0):
    tol = (2.0 ** -8 * np.abs(ref) if dtype == BF16 else 0.0) + (4e-6 + extra) * np.abs(ref).max(axis=-1, keepdims=True)
    assert np.all(np.abs(got - ref) <= tol), float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max())


def run_norm(seed, rows, d, *, dtype, stream=None, layer=False, post=False, gate="", bias=True, offset=0.0, h_scale=1.0, y_scale=1.0, mean=0.0,
             with_y=True, pad=0, in_place=False, eps=1e-5):
    stream = dtype if stream is None else stream
    rng = np.random.default_rng(seed)
    vec = lambda: plain.stored(1 - offset + 0.2 * rng.standard_normal(d), dtype)  # noqa: E731
    h, y = plain.stored(rng.standard_normal((rows, d)) * 3 + mean, stream), plain.stored(rng.standard_normal((rows, d)), dtype)
    w_pre, w_post = vec(), vec() if post else None
    b_pre, b_post = (vec(), vec() if post else None) if layer and bias else (None, None)
    g = None if not gate else plain.stored(rng.standard_normal((rows, d) if gate == "row" else d), dtype)

    def put(a, t):                           # rows `pad` elements further apart than they are long
        if a is None:
            return None
        if a.ndim == 1:
            return to_dev(a, t)
        buf = torch.full((a.shape[0], d + pad), float("nan"), dtype=torch_type(t), device="cuda")
        buf[:, :d] = to_dev(a, t)
        return buf[:, :d]

    N = G.norm(to_dev(w_pre, dtype), b_pre=to_dev(b_pre, dtype), w_post=to_dev(w_post, dtype), b_post=to_dev(b_post, dtype), eps=eps,
               w_offset=offset, kind=G.NORM_LAYER if layer else G.NORM_RMS, h_scale=h_scale, y_scale=y_scale)
    th, ty = put(h, stream), put(y, dtype)
    h_out = th if in_place else put(np.full((rows, d), 7.0), stream)
    x = ty if in_place and with_y else put(np.full((rows, d), 7.0), dtype)
    G.griffin_norm_residual(N, th, ty if with_y else None, h_out, x, gate=put(g, dtype))
    torch.cuda.synchronize()
    ref_h, ref_x = plain.norm_residual(h, y if with_y else None, g, w_pre, b_pre, w_post, b_post, layer=layer, eps=eps, offset=offset,
                                       h_scale=h_scale, y_scale=y_scale)
    norm_close(to_host(h_out), ref_h, stream)
    # a mean that is far larger than the deviations from it costs the digits that it takes
    norm_close(to_host(x), ref_x, dtype, extra=abs(mean) * 2.0 ** -22)
    if pad:
        assert bool(torch.isnan(torch.as_strided(x, (rows, pad), x.stride(), x.storage_offset() + d)).all())


@pytest.mark.parametrize("d", [8, 72, 512, 520, 2048, 2056, 4096, 5120, 8192, 8200, 16384, 16392, 32768])
@pytest.mark.parametrize("dtype,stream", [(F32, F32), (BF16, BF16), (BF16, F32)])
def test_norm_widths(d, dtype, stream):
    run_norm(d, 3, d, dtype=dtype, stream=stream, post=True, gate="d", offset=1.0, y_scale=0.25)
    run_norm(d + 1, 2, d, dtype=dtype, stream=stream, layer=True, post=True, gate="row", h_scale=0.5)


@pytest.mark.parametrize("rows", [1, 2, 5, 64, 1023])
@pytest.mark.parametrize("layer", [False, True])
def test_norm_rows(rows, layer):
    run_norm(rows, rows, 264, dtype=BF16, layer=layer, post=True)
    run_norm(rows, rows, 1032, dtype=F32, layer=layer)


@pytest.mark.parametrize("kw", [dict(with_y=False), dict(bias=False, layer=True), dict(pad=8), dict(pad=24, gate="row", post=True), dict(in_place=True),
                                dict(in_place=True, pad=16, post=True, layer=True), dict(layer=True, mean=100.0), dict(y_scale=-2.0, h_scale=0.0),
                                dict(eps=0.5)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_forms(kw, dtype):
    run_norm(11, 7, 1400, dtype=dtype, stream=F32 if kw.get("mean") else None, **kw)


def test_norm_writes_what_is_asked_for():
    d = 512
    rng = np.random.default_rng(3)
    h, y = (to_dev(plain.stored(rng.standard_normal((4, d)), BF16), BF16) for _ in range(2))
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    only_x, only_h, both = (torch.zeros_like(h) for _ in range(3))
    both_x = torch.zeros_like(h)
    N = G.norm(w, eps=1e-6)
    G.griffin_norm_residual(N, h, y, None, only_x)
    G.griffin_norm_residual(N, h, y, only_h, None)
    G.griffin_norm_residual(N, h, y, both, both_x)
    G.griffin_norm_residual(N, h[:0], y[:0], both[:0], both_x[:0])
    assert torch.equal(only_x, both_x) and torch.equal(only_h, both) and torch.equal(both, (h.float() + y.float()).bfloat16())


def test_norm_rows_that_are_not_numbers_stay_in_their_row():
    d = 1032
    h = torch.randn(6, d, device="cuda")
    h[1, 5], h[3, 1031], h[4] = float("nan"), float("inf"), 0.0
    x = torch.empty_like(h)
    G.griffin_norm_residual(G.norm(torch.ones(d, device="cuda"), eps=1e-5), h, None, None, x)
    assert bool(torch.isnan(x[1]).all()) and bool(torch.isnan(x[3, 1031])) and bool((x[3, :1031] == 0).all()) and bool((x[4] == 0).all())
    good = h[[0, 2, 5]].double()
    assert torch.allclose(x[[0, 2, 5]].double(), good / (good.square().mean(1, keepdim=True) + 1e-5).sqrt(), rtol=1e-5, atol=1e-6)


# ----------------------------------------------------------------------------------------------- the cache
def pools(c, order, gap=0):
    """device pools of a case, [page][head][slot][dim] or [page][slot][head][dim], rows `gap` elements further apart than they are long"""
    out = []
    for pool in (c.K, c.V):
        a = pool if order == "htd" else pool.transpose(0, 2, 1, 3)
        t = torch.full((*a.shape[:3], a.shape[3] + gap), float("nan"), dtype=torch_type(c.dtype), device="cuda")
        t[..., :c.dim] = dev(a, c.dtype)
        t = t[..., :c.dim]
        out.append(t if order == "htd" else t.transpose(1, 2))
    return out


def batch(c, **kw):
    return G.kv_batch(c.cu, ints(c.lens), ints(c.pages), c.max_len, prefix_pages=ints(c.prefix_pages), n_prefix=c.prefix, **kw)


def tables(n_pos, rot):
    angle = np.arange(n_pos)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def same(a, b):
    return bool(torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("heads,kv_heads,dim,rot,page,prefix,held,new,order,gap", [
    (32, 8, 128, 128, 16, 0, [0], [1], "htd", 0),
    (8, 8, 64, 64, 16, 40, [15, 16, 0, 31], [1, 1, 1, 1], "thd", 0),
    (6, 2, 80, 40, 32, 5, [0, 7, 0], [33, 0, 70], "htd", 8),             # 20 pairs: four at a time
    (4, 1, 96, 10, 64, 3, [1, -4], [5, 2], "thd", 16),                   # five pairs: one at a time; a length below zero
    (5, 5, 256, 256, 128, 0, [100], [150], "htd", 0),
    (3, 3, 8, 6, 16, 1, [2, 3], [3, 3], "htd", 0),
    (2, 1, 128, 0, 16, 9, [20], [17], "thd", 0),                         # nothing rotated
    (40, 8, 120, 64, 256, 0, [250], [12], "htd", 0),
])
def test_append(dtype, style, heads, kv_heads, dim, rot, page, prefix, held, new, order, gap):
    c = plain.Case(rot + heads, heads=heads, kv_heads=kv_heads, dim=dim, page=page, prefix=prefix, held=held, new=new, dtype=dtype)
    K, V = pools(c, order, gap)
    cos, sin = tables(prefix + c.max_len, rot)
    fused = torch.full((c.cu[-1], heads + 2 * kv_heads, dim + gap), float("nan"), dtype=torch_type(dtype), device="cuda")
    fused[..., :dim] = dev(np.concatenate([c.q, c.k, c.v], axis=1), dtype)
    q, k, v = fused[:, :heads, :dim], fused[:, heads:heads + kv_heads, :dim], fused[:, heads + kv_heads:, :dim]
    q_out = torch.full((c.cu[-1], heads, dim), 7.0, dtype=torch_type(dtype), device="cuda")
    before = K.clone(), V.clone()
    kw = dict(cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda()) if rot else {}
    kw["style"] = G.ROT_HALF if style == "half" else G.ROT_PAIRS
    G.griffin_kv_append(G.kv_cache(K, V), batch(c), k, v, q=q, q_out=q_out, **kw)
    torch.cuda.synchronize()
    want_K, want_V = np.array(c.K), np.array(c.V)
    want_q = plain.append(want_K, want_V, c.k, c.v, c.q, cos.astype(np.float64) if rot else None, sin.astype(np.float64) if rot else None,
                          style, c.cu, c.lens, c.pages, page, prefix, c.max_len)
    # values are copies, slots that nobody wrote are as they were
    assert same(V, dev(want_V, dtype))
    changed = ~(np.nan_to_num(want_K, nan=9.0) == np.nan_to_num(c.K, nan=9.0)).all(axis=-1)
    keep = torch.from_numpy(~changed).cuda()
    assert same(K[keep], before[0][keep])
    # products and a sum in fp32 (2^-24 each of at most |a| + |b| <= 10), then the output's own rounding
    for got, want in ((to_host(K), want_K), (to_host(q_out), want_q)):
        tol = (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * np.abs(want) + 10 * 2.0 ** -23
        assert np.all((np.abs(got - want) <= tol) | np.isnan(want)) and np.array_equal(np.isnan(got), np.isnan(want))
    # in place, and without queries
    K2, V2 = pools(c, order, gap)
    q2 = fused.clone()[:, :heads, :dim]
    G.griffin_kv_append(G.kv_cache(K2, V2), batch(c), k, v, q=q2, q_out=q2, **kw)
    assert torch.equal(q2, q_out) and same(K2, K)
    K2, V2 = pools(c, order, gap)
    G.griffin_kv_append(G.kv_cache(K2, V2), batch(c), k, v, **kw)
    assert same(K2, K) and same(V2, V)


def test_append_stops_at_max_len_and_clamps_pages():
    c = plain.Case(5, heads=4, kv_heads=2, dim=64, page=16, prefix=0, held=[30, 60, 64], new=[5, 8, 3], dtype=BF16, max_len=64)
    K, V = pools(c, "htd")
    pages = c.pages.copy()
    pages[0, 3] = 10 ** 6                       # not read: the sequence ends before
    B = G.kv_batch(c.cu, ints(c.lens), ints(pages), c.max_len)
    k, v, q = (dev(a, BF16) for a in (c.k, c.v, c.q))
    q_out = torch.zeros_like(q)
    G.griffin_kv_append(G.kv_cache(K, V), B, k, v, q=q, q_out=q_out)
    want_K, want_V = np.array(c.K), np.array(c.V)
    plain.append(want_K, want_V, c.k, c.v, c.q, None, None, "half", c.cu, c.lens, c.pages, 16, 0, 64)
    assert same(K, dev(want_K, BF16)) and same(V, dev(want_V, BF16)) and torch.equal(q_out, q)
    # numbers outside the pools name the first or the last page
    for number, page in ((-3, 0), (10 ** 6, c.n_pages - 1)):
        K, V = pools(c, "htd")
        one = ints([[number]])
        G.griffin_kv_append(G.kv_cache(K, V), G.kv_batch([0, 5], ints([0]), one, 16), k[:5], v[:5])
        assert torch.equal(K[page, :, :5].transpose(0, 1), k[:5])


# ----------------------------------------------------------------------------------------------- attention
# bf16: weights are rounded to bf16 for the second product (2^-8 of each, so at most 2^-8 sum p |v|), the output is rounded (2^-8 of itself, the half of a last place of 8 significant bits).
# Both types: scores are fp32 sums of up to 256 products, off by some 2^-24 x 16 (their random walk) x sum |q k| scale, which is up to 15 here:
# 1.4e-5 of the weights at worst; 3e-5 with what exp2 and the sums add.
def attention_close(got, ref, size, dtype):
    tol = (2.0 ** -8 * (size + np.abs(ref)) if dtype == BF16 else 0.0) + 3e-5 * size
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(got - ref) / np.maximum(tol, 1e-300))), np.argwhere(bad)[:4].tolist())


def run_attention(c, order="htd", gap=0, scale=None, stream=None):
    K, V = pools(c, order, gap)
    C, B = G.kv_cache(K, V), batch(c)
    q = torch.full((c.cu[-1], c.heads + 1, c.dim + gap), float("nan"), dtype=torch_type(c.dtype), device="cuda")[:, 1:, :c.dim]
    q.copy_(dev(c.q, c.dtype))
    buf = torch.full((c.cu[-1], c.heads, c.dim + gap), float("nan"), dtype=q.dtype, device="cuda")
    out = buf[..., :c.dim]
    ws = workspace(G.griffin_attention_workspace_bytes(C, B, c.heads))
    ws.fill_(0xFF)                              # NaN: nothing is read that the call has not written
    torch.cuda.synchronize()
    G.griffin_attention(C, B, q, out, scale=scale, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    assert not gap or bool(torch.isnan(buf[..., c.dim:]).all())
    return to_host(out)


def check_attention(seed, order="htd", gap=0, scale=None, **kw):
    c = plain.Case(seed, **kw)
    ref, size = c.attention(c.dim ** -0.5 if scale is None else scale)
    attention_close(run_attention(c, order, gap, scale), ref, size, c.dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads,dim,page,prefix,held,new,order,gap", [
    (4, 4, 64, 16, 0, [0], [1], "htd", 0),                               # one key
    (4, 2, 128, 16, 0, [15, 16, 17, 31, 32], [1] * 5, "htd", 0),         # ends around a tile's and a page's
    (8, 8, 128, 32, 1, [0, 3], [1, 1], "thd", 0),
    (8, 2, 128, 64, 333, [0, 100, 9], [1, 1, 1], "htd", 0),
    (6, 2, 80, 16, 50, [5, 0, 20, 3], [2, 0, 7, 1], "thd", 8),           # gaps, a sequence without new tokens
    (1, 1, 8, 16, 7, [1], [3], "htd", 0),
    (5, 1, 40, 128, 129, [127], [2], "htd", 24),
    (7, 1, 256, 16, 100, [31, 2], [1, 4], "thd", 0),
    (16, 16, 256, 32, 257, [0], [1], "htd", 0),
    (3, 3, 200, 16, 0, [64], [1], "htd", 0),
    (40, 1, 64, 16, 65, [40, 2], [1, 1], "htd", 0),                      # a group of more than 32 rows
    (12, 4, 96, 256, 1000, [3, 700], [1, 1], "htd", 0),                  # several chunks of both
    (4, 2, 128, 16, 0, [0], [100], "htd", 0),                            # a prompt
    (4, 1, 64, 32, 37, [0, 33, 5], [70, 31, 64], "thd", 0),              # prompts behind a prefix and own tokens
    (2, 2, 256, 16, 0, [0, 10], [65, 40], "htd", 0),
    (8, 4, 128, 16, 0, [-5, 0], [3, 2], "htd", 0),                       # a length below zero
])
def test_attention(dtype, heads, kv_heads, dim, page, prefix, held, new, order, gap):
    check_attention(heads + dim, order, gap, heads=heads, kv_heads=kv_heads, dim=dim, page=page, prefix=prefix, held=held, new=new, dtype=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_many_sequences(dtype):
    rng = np.random.default_rng(8)
    n = 256                                     # as many as a call takes
    check_attention(1, heads=2, kv_heads=1, dim=64, page=16, prefix=200, held=rng.integers(0, 50, n).tolist(), new=[1] * n, dtype=dtype)
    check_attention(2, heads=4, kv_heads=2, dim=128, page=16, prefix=20, held=rng.integers(0, 40, 60).tolist(), new=rng.integers(0, 6, 60).tolist(),
                    dtype=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_long_caches(dtype):
    check_attention(4, heads=2, kv_heads=1, dim=64, page=64, prefix=20000, held=[0, 5000], new=[1, 1], dtype=dtype)
    check_attention(5, heads=1, kv_heads=1, dim=128, page=256, prefix=0, held=[30000], new=[1], dtype=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale,q_scale", [(1e-3, 1.0), (0.5, 4.0), (8.0, 4.0)])
def test_attention_of_flat_and_sharp_scores(dtype, scale, q_scale):
    """With a large scale one key takes nearly all of a row's weight, and scores are in the hundreds; their error grows with them."""
    c = plain.Case(21, heads=4, kv_heads=2, dim=64, page=16, prefix=150, held=[70, 3], new=[2, 1], dtype=dtype, q_scale=q_scale)
    ref, size = c.attention(scale)
    got = run_attention(c, scale=scale)
    # 2^-24 x 16 x sum |q k| scale, and the rounding of s log2(e): sum |q k| is some 0.64 x 64 x q_scale
    extra = 2.0 ** -24 * 20 * 0.64 * 64 * q_scale * scale * 2
    tol = (2.0 ** -8 * (size + np.abs(ref)) if dtype == BF16 else 0.0) + (3e-5 + extra) * size.max()
    assert np.all(np.abs(got - ref) <= tol)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_keeps_what_later_tokens_hold_from_earlier_ones(dtype, dim):
    """NaN and infinities in the key or value of a new token reach the tokens that see it and no others."""
    c = plain.Case(31, heads=4, kv_heads=2, dim=dim, page=16, prefix=0, held=[3, 30], new=[40, 9], dtype=dtype)
    ref, size = c.attention(dim ** -0.5)
    at = lambda b, i: (c.pages[b, i // 16], i % 16)  # noqa: E731
    page, slot = at(0, 3 + 25)
    c.K[page, 0, slot] = np.nan                 # kv head 0: keys not a number from the sequence's token 25 on
    page, slot = at(0, 3 + 10)
    c.V[page, 1, slot, 5], c.V[page, 1, slot, 6], c.V[page, 1, slot, dim - 1] = np.inf, -np.inf, np.nan
    page, slot = at(1, 30 + 8)
    c.V[page, 0, slot, 0] = np.inf              # the last token's own
    got = run_attention(c)
    want = ref.copy()
    want[25:40, 0:2] = np.nan
    want[10:40, 2:4, 5], want[10:40, 2:4, 6], want[10:40, 2:4, dim - 1] = np.inf, -np.inf, np.nan
    want[48, 0:2, 0] = np.inf
    odd = ~np.isfinite(want)
    assert np.array_equal(np.nan_to_num(got[odd], nan=1, posinf=2, neginf=3), np.nan_to_num(want[odd], nan=1, posinf=2, neginf=3))
    attention_close(np.where(odd, 0, got), np.where(odd, 0, want), size, dtype)


def test_attention_of_scores_that_are_all_minus_infinity():
    c = plain.Case(41, heads=1, kv_heads=1, dim=64, page=16, prefix=0, held=[4], new=[1], dtype=F32)
    c.q[:] = 1.0
    c.K[c.pages[0, 0], 0, :5] = 0.0
    c.K[c.pages[0, 0], 0, :5, 0] = -np.inf
    assert np.array_equal(run_attention(c), np.zeros((1, 1, 64)))
    c.K[c.pages[0, 0], 0, 2, 0] = 1.0           # one key is left
    assert np.array_equal(run_attention(c)[0, 0], c.V[c.pages[0, 0], 0, 2])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_beyond_max_len(dtype):
    """Own tokens from max_len on are neither stored nor read, and page numbers outside the pools are clamped."""
    check_attention(51, heads=2, kv_heads=2, dim=64, page=16, prefix=10, held=[30, 20, 60], new=[4, 30, 2], dtype=dtype, max_len=33)
    c = plain.Case(52, heads=2, kv_heads=1, dim=64, page=16, prefix=0, held=[20, 20], new=[1, 1], dtype=dtype)
    ref, size = c.attention(0.125)
    c.pages[1] = [-7, 2 ** 31 - 1]
    got = run_attention(c)                      # sequence 1 reads pages of NaN or of others; sequence 0 is as it was
    attention_close(got[:1], ref[:1], size[:1], dtype)


def test_attention_offsets_past_32_bits():
    """A page whose elements begin beyond 2^31 elements and 2^32 bytes."""
    c = plain.Case(61, heads=4, kv_heads=2, dim=128, page=16, prefix=20, held=[20], new=[1], dtype=BF16)
    ref, size = c.attention(128 ** -0.5)
    far = 2 ** 31 // (2 * 16 * 128) + 5         # pages
    pool = torch.empty((far + c.n_pages, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    both = [pool, torch.empty_like(pool)]
    for big, small in zip(both, (c.K, c.V)):
        big[far:] = dev(small, BF16)
    C = G.kv_cache(*both)
    B = G.kv_batch(c.cu, ints(c.lens), ints(c.pages + far), c.max_len, prefix_pages=ints(c.prefix_pages + far), n_prefix=c.prefix)
    q = dev(c.q, BF16)
    out = torch.empty_like(q)
    G.griffin_attention(C, B, q, out, workspace=workspace(G.griffin_attention_workspace_bytes(C, B, 4)))
    attention_close(to_host(out), ref, size, BF16)
    k, v = dev(c.k, BF16), dev(c.v, BF16)
    G.griffin_kv_append(C, B, k, v)
    page = int(c.pages[0, 1]) + far
    assert torch.equal(both[0][page, :, 4], k[0]) and torch.equal(both[1][page, :, 4], v[0])


def test_step_on_another_stream_and_in_a_graph():
    """Append and attention of three steps on a side stream, then captured once and replayed: lengths are read on the device."""
    c = plain.Case(71, heads=4, kv_heads=2, dim=64, page=16, prefix=40, held=[14, 40], new=[1, 1], dtype=BF16, max_len=60)
    for b in range(2):
        c.pages[b, :4] = np.arange(4) + c.n_pages + 4 * b           # pages of their own for all that is to come
    blank = np.zeros((8, 2, 16, 64))
    c.K, c.V = (np.nan_to_num(np.concatenate([p, blank])) for p in (c.K, c.V))
    c.n_pages += 8
    K, V = pools(c, "htd")
    steps = 5
    rng = np.random.default_rng(9)
    new = [plain.stored(rng.standard_normal((steps, 2, n, 64)), BF16) for n in (4, 2, 2)]
    cos, sin = tables(c.prefix + c.max_len, 64)
    tc, ts = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    lens = ints(c.lens)
    B = G.kv_batch(c.cu, lens, ints(c.pages), c.max_len, prefix_pages=ints(c.prefix_pages), n_prefix=c.prefix)
    C = G.kv_cache(K, V)
    q, k, v = (dev(a[0], BF16) for a in new)
    q_rot, out = torch.zeros_like(q), torch.zeros_like(q)
    ws = workspace(G.griffin_attention_workspace_bytes(C, B, 4))

    def step():
        G.griffin_kv_append(C, B, k, v, q=q, q_out=q_rot, cos=tc, sin=ts)
        G.griffin_attention(C, B, q_rot, out, workspace=ws)
        lens.add_(1)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    for i in range(steps):
        for t, a in zip((q, k, v), new):
            t.copy_(dev(a[i], BF16))
        torch.cuda.synchronize()
        if i < 2:
            with torch.cuda.stream(side):
                step()
        elif i == 2:
            with torch.cuda.graph(graph, stream=side):
                step()
        if i >= 2:
            graph.replay()
        torch.cuda.synchronize()
        c.q = plain.append(c.K, c.V, *(new[j][i] for j in (1, 2, 0)), cos.astype(np.float64), sin.astype(np.float64), "half", c.cu, c.lens, c.pages,
                           16, c.prefix, c.max_len)
        c.q, c.K = plain.stored(c.q, BF16), plain.stored(c.K, BF16)
        ref, size = c.attention(0.125)
        # rotated queries and keys may round the other way where fp32 and 64 bits differ: an element in some thousands, by 2^-8 of itself
        assert np.abs(to_host(out) - ref).max() <= 0.02 * size.max(), i
        c.lens = [n + 1 for n in c.lens]
    assert lens.tolist() == c.lens


def test_results_do_not_depend_on_the_run():
    c = plain.Case(81, heads=8, kv_heads=2, dim=128, page=16, prefix=700, held=[30, 2, 9], new=[1, 1, 1], dtype=BF16)
    first = run_attention(c)
    for _ in range(3):
        assert np.array_equal(run_attention(c), first)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_own_parts_a_wavefront_each(dtype):
    """Enough sequences and heads that own parts are not shared between wavefronts: with a prefix and without, one chunk and several, a few new tokens."""
    rng = np.random.default_rng(12)
    check_attention(91, heads=8, kv_heads=8, dim=64, page=16, prefix=0, held=rng.integers(0, 33, 200).tolist(), new=[1] * 200, dtype=dtype, max_len=128)
    check_attention(92, heads=16, kv_heads=8, dim=64, page=32, prefix=45, held=rng.integers(0, 300, 64).tolist(), new=rng.integers(0, 3, 64).tolist(),
                    dtype=dtype, order="thd")
    check_attention(93, heads=16, kv_heads=16, dim=128, page=16, prefix=3, held=rng.integers(0, 150, 64).tolist(), new=[1] * 64, dtype=dtype)
    check_attention(94, heads=8, kv_heads=8, dim=256, page=16, prefix=20, held=rng.integers(0, 150, 120).tolist(), new=[1] * 120, dtype=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_of_ragged_prompts(dtype, dim):
    """Packed prompts of no, one and several tiles of rows, in no order of their lengths, behind own tokens and a prefix."""
    rng = np.random.default_rng(13)
    new = [0, 1, 300, 64, 0, 129, 5, 65, 257, 30, 128, 2]
    check_attention(95, heads=4, kv_heads=2, dim=dim, page=16, prefix=70, held=rng.integers(0, 90, len(new)).tolist(), new=new, dtype=dtype)
    check_attention(96, heads=2, kv_heads=2, dim=dim, page=64, prefix=0, held=[0] * len(new), new=new, dtype=dtype, order="thd")


def test_attention_of_a_prompt_alone_and_row_by_row():
    """Tokens of a prompt in one call and one a call give the same within their roundings: every row sees the same keys either way."""
    c = plain.Case(97, heads=4, kv_heads=2, dim=128, page=16, prefix=33, held=[20], new=[90], dtype=BF16)
    whole = run_attention(c)
    ref, size = c.attention(128 ** -0.5)
    attention_close(whole, ref, size, BF16)
    for i in (0, 1, 31, 63, 89):
        one = plain.Case(97, heads=4, kv_heads=2, dim=128, page=16, prefix=33, held=[20], new=[90], dtype=BF16)
        one.q, one.lens, one.new, one.cu = c.q[i:i + 1], [20 + i], [1], [0, 1]
        attention_close(run_attention(one), ref[i:i + 1], size[i:i + 1], BF16)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("prefix", [1, 64, 70])
def test_attention_of_prompts_that_fill_the_chip_behind_a_prefix(dim, prefix):
    """Enough tiles of rows that each takes the prefix ahead of its own keys (bf16), the prefix ending in a tile of 16 keys and at its end."""
    check_attention(98 + dim, heads=32, kv_heads=32, dim=dim, page=16, prefix=prefix, held=[0, 17, 3, 0], new=[260, 300, 70, 259] if dim <= 128 else [130, 150, 70, 129],
                    dtype=BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads,new", [(4, 2, [1, 3]), (32, 32, [260, 257])])
def test_attention_of_infinities_beside_the_prefix_end(dtype, heads, kv_heads, new):
    """An infinite value in the 16 keys in which the prefix ends, and NaN behind its last token: one reaches everybody, the other nobody."""
    c = plain.Case(99, heads=heads, kv_heads=kv_heads, dim=64, page=32, prefix=37, held=[2, 9], new=new, dtype=dtype)
    ref, size = c.attention(0.125)
    assert np.isnan(c.V[c.prefix_pages[1], 0, 5]).all()
    c.V[c.prefix_pages[1], 1, 3, 7] = -np.inf
    got = run_attention(c, scale=0.125)
    group = heads // kv_heads
    assert np.all(got[:, group:2 * group, 7] == -np.inf)
    got[:, group:2 * group, 7], ref[:, group:2 * group, 7] = 0, 0
    attention_close(got, ref, size, dtype)


@pytest.mark.parametrize("heads,kv_heads,dim,prefix,held,new,order", [
    (128, 4, 80, 23500, [0, 600, 33, 270, 5, 9, 256, 1, 300], [1] * 9, "thd"),        # a workgroup each, two tiles of rows, several chunks of own parts
    (64, 2, 128, 43700, [700, 0, 250], [1, 3, 2], "htd"),                             # ... of up to 96 rows: own parts are tiles, too
    (64, 2, 128, 43700, [700, 0, 250, 3, 31], [1, 1, 1, 2, 1], "htd"),                # ... of up to 64
    (128, 16, 64, 4200, list(range(0, 192, 3)), [1] * 64, "htd"),                     # a wavefront each
])
def test_attention_of_own_parts_beside_tiles_of_the_prefix(heads, kv_heads, dim, prefix, held, new, order):
    """bf16: a prefix with so much to multiply that its rows go in tiles, own parts of a few rows behind them."""
    assert sum(new) * heads * dim * prefix >= 2 ** 31
    check_attention(111, order, heads=heads, kv_heads=kv_heads, dim=dim, page=64, prefix=prefix, held=held, new=new, dtype=BF16)
