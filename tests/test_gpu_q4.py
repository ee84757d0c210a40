"""The cache in 4 bits (append, read, attention) against its definitions in 64 bits."""
import numpy as np
import pytest
import torch

import layer_plain as plain
import paper_2404_01365_amd as G
import q4_plain
import synth
from devio import to_host, workspace
from test_gpu_layer import dev, ints, tables, torch_type

pytestmark = pytest.mark.gpu

F32, BF16 = synth.DT_F32, synth.DT_BF16


def put(pool):
    return torch.from_numpy(pool).cuda()


def cache(c, K, V, group):
    return G.kv_cache_q4(K, V, kv_heads=c.kv_heads, dim=c.dim, page_size=c.page, group=group, dtype=torch_type(c.dtype))


def batch(c, **kw):
    return G.kv_batch(c.cu, ints(c.lens), ints(c.pages), c.max_len, prefix_pages=ints(c.prefix_pages), n_prefix=c.prefix, **kw)


def spread(a, dtype, gap):
    """[tokens][heads][dim] with `gap` elements between the heads' rows and a head between the tokens'"""
    buf = torch.full((a.shape[0], a.shape[1] + 1, a.shape[2] + gap), float("nan"), dtype=torch_type(dtype), device="cuda")
    buf[:, 1:, :a.shape[2]] = dev(a, dtype)
    return buf[:, 1:, :a.shape[2]]


# ----------------------------------------------------------------------------------------------- append
def run_append(c, group, style, rot, gap=0, fill=0xA5, in_place=False):
    size = q4_plain.page_bytes(c.kv_heads, c.dim, c.page, group)
    pools = [np.full((c.n_pages, size), fill, np.uint8) for _ in range(2)]
    K, V = (put(x) for x in pools)
    cos = sin = None
    if rot:
        cos, sin = (np.asarray(t, np.float32) for t in tables(c.prefix + c.max_len, rot))
    q = spread(c.q, c.dtype, gap)
    q_out = q if in_place else torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    on = lambda t: None if t is None else torch.from_numpy(t).cuda()  # noqa: E731
    G.griffin_kv_append_q4(cache(c, K, V, group), batch(c), spread(c.k, c.dtype, gap), spread(c.v, c.dtype, gap), q=q, q_out=q_out, cos=on(cos), sin=on(sin),
                           style=G.ROT_HALF if style == "half" else G.ROT_PAIRS)
    torch.cuda.synchronize()
    views = [v for x in pools for v in q4_plain.parts(x, c.kv_heads, c.dim, c.page, group)]
    flat = [np.array(v) for v in views]
    q4_plain.append(flat[0], flat[1], flat[2], flat[3], c, cos, sin, style, group)
    # the plain result as bytes: the pools are untouched but for the step's rows, and those are the definition's bit for bit
    for got, codes, pairs in ((K, flat[0], flat[1]), (V, flat[2], flat[3])):
        got_codes, got_pairs = q4_plain.parts(got.cpu().numpy(), c.kv_heads, c.dim, c.page, group)
        got_pairs, pairs = (np.ascontiguousarray(x).view(np.uint16) for x in (got_pairs, pairs))
        for a, b in ((got_codes, codes), (got_pairs, pairs)):
            off = np.argwhere(a != b)
            assert len(off) == 0, (len(off), off[:3].tolist(), [(int(a[tuple(i)]), int(b[tuple(i)])) for i in off[:3]])
    return q_out, cos, sin


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("heads,kv_heads,dim,rot,page,prefix,held,new,group,gap", [
    (4, 2, 64, 64, 16, 0, [0], [1], 32, 0),
    (8, 2, 128, 128, 64, 100, [0, 15, 200], [1, 1, 1], 32, 0),
    (8, 8, 128, 64, 16, 7, [3, 0, 31], [5, 0, 40], 64, 8),               # ragged, half of the features rotated
    (5, 5, 80, 80, 32, 0, [9, 2], [3, 3], 32, 0),                        # a last group of 16, halves of 40
    (3, 1, 96, 0, 16, 3, [0], [20], 64, 16),                             # nothing rotated, a last group of 32
    (2, 1, 40, 20, 16, 1, [0, 3], [2, 1], 64, 0),                        # pairs at odd places
    (2, 2, 8, 6, 16, 0, [15], [2], 32, 0),
    (7, 1, 256, 256, 128, 50, [127, 0], [2, 130], 32, 8),
    (4, 4, 200, 100, 16, 0, [16], [17], 64, 0),
])
def test_append(dtype, style, heads, kv_heads, dim, rot, page, prefix, held, new, group, gap):
    c = plain.Case(dim + rot, heads=heads, kv_heads=kv_heads, dim=dim, page=page, prefix=prefix, held=held, new=new, dtype=dtype)
    for in_place in (False, True):
        q_out, cos, sin = run_append(c, group, style, rot, gap, in_place=in_place)
        got = to_host(q_out)
        for t in range(c.cu[-1]):
            b = int(np.searchsorted(c.cu, t, side="right")) - 1
            pos = prefix + held[b] + t - c.cu[b]
            want = plain.rotate(c.q[t], cos[pos].astype(np.float64), sin[pos].astype(np.float64), style) if rot else c.q[t]
            # fp32: two products and a sum of numbers below 8, rounded to half a last place each; bf16: the output's rounding
            tol = 3 * 2.0 ** -24 * 2 * np.abs(c.q[t]).max() + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0)
            assert np.all(np.abs(got[t] - want) <= tol)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", [32, 64])
def test_append_of_values_that_stand_out(dtype, group):
    c = plain.Case(3, heads=2, kv_heads=2, dim=128, page=16, prefix=0, held=[0], new=[14], dtype=dtype)
    t = c.k
    t[0, 0, 5] = np.nan                      # a group that is not finite, its neighbours as ever
    t[1, 1, 70], t[2, 0, 127] = np.inf, -np.inf
    t[3] = 0.0
    t[4] = plain.stored(1.7, dtype)          # no spread: the middle alone
    t[5, :, :40] = plain.stored(-3e38, F32 if dtype == F32 else BF16)
    t[6, 0, 3], t[6, 1, 3] = 1e30, -40000.0  # cut to the format's range
    t[7] *= plain.stored(2.0 ** -20, dtype)  # scales below fp16's normal numbers
    t[8] *= 2.0 ** -30                       # ... and none at all
    t[9] = 1000 + t[9] * 2.0 ** -4 if dtype == F32 else t[9] * 4096
    t[10, 0] = np.arange(128) % 16 - 8.0     # whole steps: every code, and ties of none
    t[11, 0] = (np.arange(128) % 31 - 15) / 2.0
    t[12, :, 0] = 32768.0
    t[13, :, ::2], t[13, :, 1::2] = 65536.0, -65536.0
    c.k = plain.stored(t, dtype)
    c.v = np.array(c.k[::-1])
    run_append(c, group, "half", 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", [32, 64])
def test_append_of_middles_at_zero(dtype, group):
    """groups whose middle is zero, or next to it, and nothing else: zero's sign is the definition's, too"""
    c = plain.Case(8, heads=2, kv_heads=2, dim=128, page=16, prefix=0, held=[0], new=[40], dtype=dtype)
    steps = (np.arange(128) % 16 - 8.0)[None, None, :] * 2.0 ** (np.arange(40) % 12 - 6)[:, None, None]
    c.k = plain.stored(np.broadcast_to(steps, c.k.shape), dtype)
    c.v = np.array(-c.k)
    run_append(c, group, "half", 0)


def test_append_stops_at_max_len_and_clamps_pages():
    c = plain.Case(5, heads=4, kv_heads=2, dim=64, page=16, prefix=0, held=[30, 60, 64, -7], new=[5, 8, 3, 2], dtype=BF16, max_len=64)
    run_append(c, 32, "half", 64)
    size = q4_plain.page_bytes(2, 64, 16, 32)
    for number, page in ((-3, 0), (10 ** 6, 4)):
        K, V = (torch.full((5, size), 7, dtype=torch.uint8, device="cuda") for _ in range(2))
        C = G.kv_cache_q4(K, V, kv_heads=2, dim=64, page_size=16, dtype=torch.bfloat16)
        k = dev(c.k[:5], BF16)
        G.griffin_kv_append_q4(C, G.kv_batch([0, 5], ints([0]), ints([[number]]), 16), k, k)
        assert bool((K[page] != 7).any())
        K[page] = 7
        assert bool((K == 7).all())


# ----------------------------------------------------------------------------------------------- read
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kv_heads,dim,page,held,new,group,gap", [
    (2, 64, 16, [0], [1], 32, 0), (8, 128, 64, [3, 0, 100], [5, 0, 70], 64, 8), (5, 80, 16, [9], [33], 32, 0), (3, 96, 32, [1, 1], [40, 2], 64, 8),
    (1, 8, 16, [15], [3], 32, 0), (2, 256, 128, [0, 7], [150, 1], 32, 0), (4, 200, 16, [5], [30], 64, 16)])
def test_read(dtype, kv_heads, dim, page, held, new, group, gap):
    c = plain.Case(dim, heads=kv_heads, kv_heads=kv_heads, dim=dim, page=page, prefix=0, held=held, new=new, dtype=dtype)
    K, V = (q4_plain.pool_of(x * 3, group) for x in (c.K, c.V))
    C, B = cache(c, put(K), put(V), group), batch(c)
    want = []
    for pool in (K, V):
        all_of = q4_plain.values(*q4_plain.parts(pool, kv_heads, dim, page, group), dim, group)
        rows = [all_of[c.pages[b, (held[b] + i) // page], :, (held[b] + i) % page] for b in range(len(new)) for i in range(new[b])]
        want.append(dev(np.stack(rows), dtype))
    k, v = spread(np.zeros((c.cu[-1], kv_heads, dim)), dtype, gap), torch.zeros(c.cu[-1], kv_heads, dim, dtype=torch_type(dtype), device="cuda")
    G.griffin_kv_read_q4(C, B, k, v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    k.zero_(), v.zero_()
    G.griffin_kv_read_q4(C, B, v=v)
    assert torch.equal(v, want[1]) and not k.any()
    G.griffin_kv_read_q4(C, B, k)
    assert torch.equal(k, want[0])


def test_read_beyond_max_len_leaves_rows_as_they_were():
    c = plain.Case(4, heads=2, kv_heads=2, dim=64, page=16, prefix=0, held=[14, -2], new=[6, 3], dtype=F32, max_len=17)
    K, V = (put(q4_plain.pool_of(x, 32)) for x in (c.K, c.V))
    k, v = (torch.full((9, 2, 64), 5.0, device="cuda") for _ in range(2))
    G.griffin_kv_read_q4(cache(c, K, V, 32), batch(c), k, v)
    assert bool((k[3:6] == 5).all()) and bool((v[3:6] == 5).all()) and not bool((k[:3] == 5).any()) and not bool((v[6:] == 5).any())


def test_what_is_appended_is_read_back():
    """Prompt, prefix and a step through the public calls alone; half a step of every group off at most."""
    c = plain.Case(9, heads=8, kv_heads=4, dim=128, page=32, prefix=0, held=[0, 5], new=[70, 9], dtype=F32)
    size = G.griffin_kv_q4_page_bytes(4, 128, 32, 64)
    K, V = (torch.zeros(c.n_pages, size, dtype=torch.uint8, device="cuda") for _ in range(2))
    C, B = cache(c, K, V, 64), batch(c)
    k, v = dev(c.k, F32), dev(c.v, F32)
    G.griffin_kv_append_q4(C, B, k, v)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    G.griffin_kv_read_q4(C, B, k2, v2)
    for x, y in ((k, k2), (v, v2)):
        g = x.unflatten(2, (2, 64))
        step = (g.amax(dim=3) - g.amin(dim=3)) / 15
        tol = step[..., None] / 2 + 2.0 ** -11 * (g.abs().amax(dim=3) + 8 * step)[..., None]
        assert bool(((y.unflatten(2, (2, 64)) - g).abs() <= tol).all())


# ----------------------------------------------------------------------------------------------- attention
# Keys, values and bf16 queries enter exactly.  Weights are cut to fp16, at most 2^-10 of each, in numerator and denominator: 2^-10 (sum p |v| + |out|); fp32 caches take two fp16 for
# a weight, 2^-20, and for a query, 2^-23 of each product, which a score of sum |q k| scale up to 15 is off by 1.8e-6 for.  Scores are fp32 sums of up to 256 products, off by
# some 2^-24 x 16 x sum |q k| scale (their random walk): 1.4e-5 of the weights; with exp2 and the sums 3e-5.  A bf16 output adds its rounding, 2^-8 of itself.
def attention_close(got, ref, size, dtype, extra=0.0):
    tol = (2.0 ** -10 * (size + np.abs(ref)) + 2.0 ** -8 * np.abs(ref) if dtype == BF16 else 2.0 ** -20 * (size + np.abs(ref))) + (3e-5 + extra) * size
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(got - ref) / np.maximum(tol, 1e-300))), np.argwhere(bad)[:4].tolist())


def run_attention(c, K, V, group, gap=0, scale=None, stream=None):
    C, B = cache(c, put(K), put(V), group), batch(c)
    q = spread(c.q, c.dtype, gap)
    buf = torch.full((c.cu[-1], c.heads, c.dim + gap), float("nan"), dtype=q.dtype, device="cuda")
    out = buf[..., :c.dim]
    ws = workspace(G.griffin_attention_q4_workspace_bytes(C, B, c.heads))
    ws.fill_(0xFF)                              # NaN: nothing is read that the call has not written
    torch.cuda.synchronize()
    G.griffin_attention_q4(C, B, q, out, scale=scale, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    assert not gap or bool(torch.isnan(buf[..., c.dim:]).all())
    return to_host(out)


def reference(c, K, V, group, scale):
    c.K, c.V = (q4_plain.values(*q4_plain.parts(x, c.kv_heads, c.dim, c.page, group), c.dim, group) for x in (K, V))
    return c.attention(c.dim ** -0.5 if scale is None else scale)


def check_attention(seed, group=32, gap=0, scale=None, size=1.0, **kw):
    c = plain.Case(seed, **kw)
    K, V = q4_plain.pool_of(c.K, group), q4_plain.pool_of(c.V * size, group)
    ref, most = reference(c, K, V, group, scale)
    attention_close(run_attention(c, K, V, group, gap, scale), ref, most, c.dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads,dim,page,prefix,held,new,group,gap", [
    (4, 4, 64, 16, 0, [0], [1], 32, 0),                                  # one key
    (4, 2, 128, 16, 0, [15, 16, 17, 31, 32], [1] * 5, 32, 0),            # ends around a tile's and a page's
    (8, 8, 128, 32, 1, [0, 3], [1, 1], 64, 0),
    (8, 2, 128, 64, 333, [0, 100, 9], [1, 1, 1], 32, 0),
    (6, 2, 80, 16, 50, [5, 0, 20, 3], [2, 0, 7, 1], 32, 8),              # gaps, a sequence without new tokens
    (1, 1, 8, 16, 7, [1], [3], 32, 0),
    (5, 1, 40, 128, 129, [127], [2], 64, 24),
    (7, 1, 256, 16, 100, [31, 2], [1, 4], 32, 0),
    (16, 16, 256, 32, 257, [0], [1], 64, 0),
    (3, 3, 200, 16, 0, [64], [1], 32, 0),
    (2, 1, 160, 16, 33, [16], [2], 32, 0),
    (40, 1, 64, 16, 65, [40, 2], [1, 1], 32, 0),                         # a group of more than 32 rows
    (12, 4, 96, 256, 1000, [3, 700], [1, 1], 64, 0),                     # several chunks of both
    (4, 2, 128, 16, 0, [0], [100], 32, 0),                               # a prompt
    (4, 1, 64, 32, 37, [0, 33, 5], [70, 31, 64], 64, 0),                 # prompts behind a prefix and own tokens
    (2, 2, 256, 16, 0, [0, 10], [65, 40], 32, 0),
    (8, 4, 128, 16, 0, [-5, 0], [3, 2], 32, 0),                          # a length below zero
])
def test_attention(dtype, heads, kv_heads, dim, page, prefix, held, new, group, gap):
    check_attention(heads + dim, group, gap, heads=heads, kv_heads=kv_heads, dim=dim, page=page, prefix=prefix, held=held, new=new, dtype=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_many_sequences(dtype):
    rng = np.random.default_rng(8)
    n = 256                                     # as many as a call takes
    check_attention(1, heads=2, kv_heads=1, dim=64, page=16, prefix=200, held=rng.integers(0, 50, n).tolist(), new=[1] * n, dtype=dtype)
    check_attention(2, heads=4, kv_heads=2, dim=128, page=16, prefix=20, held=rng.integers(0, 40, 60).tolist(), new=rng.integers(0, 6, 60).tolist(),
                    dtype=dtype)
    check_attention(3, heads=32, kv_heads=32, dim=64, page=16, prefix=0, held=rng.integers(0, 200, 40).tolist(), new=[1] * 40, dtype=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_long_caches(dtype):
    check_attention(4, heads=2, kv_heads=1, dim=64, page=64, prefix=20000, held=[0, 5000], new=[1, 1], dtype=dtype)
    check_attention(5, heads=1, kv_heads=1, dim=128, page=256, prefix=0, held=[30000], new=[1], dtype=dtype, group=64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_of_drafts_and_ragged_prompts(dtype, dim):
    check_attention(6, heads=8, kv_heads=2, dim=dim, page=32, prefix=700, held=[3, 90, 0, 41], new=[5, 5, 5, 5], dtype=dtype)
    check_attention(7, heads=4, kv_heads=2, dim=dim, page=16, prefix=0, held=[0, 7, 0, 100], new=[130, 1, 0, 67], dtype=dtype, group=64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [40, 64, 96, 128, 200, 256])
def test_attention_of_ragged_prompts(dtype, dim):
    check_attention(13, heads=10, kv_heads=2, dim=dim, page=16, prefix=0, held=[0, 3, 0, 40, 0, 9], new=[150, 70, 13, 64, 0, 129], dtype=dtype)
    check_attention(14, heads=4, kv_heads=1, dim=dim, page=32, prefix=77, held=[0, 3, 0, 250], new=[160, 70, 33, 64], dtype=dtype, group=64)


def test_attention_of_a_prompt_alone_and_row_by_row():
    """The rows of a prompt in one call (through LDS) and one token a call (straight from memory)"""
    c = plain.Case(15, heads=8, kv_heads=2, dim=128, page=16, prefix=0, held=[0], new=[90], dtype=BF16)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    together = run_attention(c, K, V, 32)
    for i in (0, 1, 31, 32, 63, 64, 89):
        one = plain.Case(15, heads=8, kv_heads=2, dim=128, page=16, prefix=0, held=[0], new=[90], dtype=BF16)
        one.q, one.cu, one.lens = c.q[i:i + 1], [0, 1], [i]
        alone = run_attention(one, K, V, 32)[0]
        # the output's rounding to bf16 twice, and weights that are cut apart from each other, 2^-10 of values below 5
        assert np.all(np.abs(alone - together[i]) <= 2.0 ** -7 * np.abs(alone) + 2.0 ** -10 * 2 * 5)


@pytest.mark.parametrize("heads,kv_heads,dim,prefix,held,new", [
    (32, 8, 128, 0, 30000, 1100),           # 35 tiles of a kv head, parts in three rounds
    (16, 4, 64, 0, 20000, 3000),            # more tiles than a round takes, cut
    (32, 8, 128, 30000, 0, 700),            # a prefix in several rounds, own parts of one
    (16, 8, 256, 9000, 7000, 700)])
def test_attention_of_prompts_in_several_rounds_and_row_by_row(heads, kv_heads, dim, prefix, held, new):
    """a long prompt on a long cache (through LDS, in more parts than workgroups fit the chip) and one token a call (straight from memory)"""
    page, g = 128, torch.Generator(device="cuda")
    g.manual_seed(dim + new)
    keys = -(-prefix // page) * page + held + new
    n = -(-keys // page)
    size = G.griffin_kv_q4_page_bytes(kv_heads, dim, page)
    K, V = (torch.zeros(n, size, dtype=torch.uint8, device="cuda") for _ in range(2))
    C = G.kv_cache_q4(K, V, kv_heads=kv_heads, dim=dim, page_size=page, dtype=torch.bfloat16)
    k, v = (torch.empty(keys, kv_heads, dim, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    q = torch.empty(new, heads, dim, dtype=torch.bfloat16, device="cuda").normal_(generator=g) * 2
    numbers = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[None]
    G.griffin_kv_append_q4(C, G.kv_batch([0, keys], ints([0]), numbers, n * page), k, v)       # the prefix's pages, then the sequence's
    first = -(-prefix // page)
    pages, shared = numbers[:, first:].contiguous(), numbers[0, :first].contiguous()

    def run(rows, at, max_len):
        B = G.kv_batch([0, rows.shape[0]], ints([at]), pages, max_len, prefix_pages=shared, n_prefix=prefix)
        out = torch.full_like(rows, float("nan"))
        ws = workspace(G.griffin_attention_q4_workspace_bytes(C, B, heads))
        ws.fill_(0xFF)
        G.griffin_attention_q4(C, B, rows, out, workspace=ws)
        return to_host(out)

    together = run(q, held, held + new)
    most = float(v.abs().max())
    for i in (0, 1, 31, 32, 63, 64, 500, new - 1):
        alone = run(q[i:i + 1], held + i, held + new)[0]
        # the output's rounding to bf16 twice, and weights that are cut apart from each other, 2^-10 of the values
        assert np.all(np.abs(alone - together[i]) <= 2.0 ** -7 * np.abs(alone) + 2.0 ** -10 * 2 * most)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("prefix", [1, 64, 70])
def test_attention_of_prompts_that_fill_the_chip_behind_a_prefix(dim, prefix):
    check_attention(16, heads=28, kv_heads=28, dim=dim, page=16, prefix=prefix, held=[0, 20, 5], new=[130, 257, 270], dtype=BF16)


@pytest.mark.parametrize("heads,kv_heads,dim,prefix,held,new", [
    (64, 2, 128, 25000, [0, 300, 31, 700, 64, 200, 7, 90, 3], [1, 1, 1, 2, 1, 1, 1, 1, 2]),      # 352 rows a kv head, own parts a workgroup each, cut by the device
    (64, 2, 128, 25000, [0, 30, 31, 70, 64, 20, 7, 90, 3], [1, 1, 1, 2, 1, 1, 1, 1, 2]),         # ... too short to be cut
    (16, 8, 64, 20000, [int(x) for x in np.random.default_rng(3).integers(0, 200, 130)], [1] * 130),     # ... a wavefront each
    (80, 1, 96, 71000, [0, 9, 600], [1, 1, 2]),
    (48, 1, 256, 45000, [30, 1], [3, 1])])                                                         # own parts in a launch of their own
def test_attention_of_own_parts_beside_tiles_of_the_prefix(heads, kv_heads, dim, prefix, held, new):
    check_attention(17, heads=heads, kv_heads=kv_heads, dim=dim, page=64, prefix=prefix, held=held, new=new, dtype=BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_groups_of_nan_in_prompts_behind_a_prefix(dtype, dim):
    """... in the prefix (everyone sees them), beside the place where it ends, and among a prompt's own keys"""
    c = plain.Case(18, heads=32, kv_heads=32, dim=dim, page=16, prefix=21, held=[0, 6], new=[260, 40], dtype=dtype)
    clean = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, size = reference(c, *clean, 32, None)
    V = np.array(clean[1])
    row, groups = q4_plain.sizes(dim, 32)

    def spoil(page, slot, head, g):
        V.reshape(V.shape[0], 32, -1)[page, head][16 * row:].view(np.float16).reshape(16, groups, 2)[slot, g] = np.float16(np.nan), np.float16(0)

    spoil(c.prefix_pages[1], 4, 3, 0)                    # the prefix's last key
    for i, head, g in ((0, 5, 1), (200, 7, 0), (259, 9, groups - 1)):
        spoil(c.pages[0, i // 16], i % 16, head, g)
    spoil(c.pages[1, (6 + 39) // 16], (6 + 39) % 16, 11, 0)
    got = run_attention(c, clean[0], V, 32)
    want = ref.copy()
    want[:, 3, :32] = np.nan
    want[0:260, 5, 32:64] = want[200:260, 7, :32] = want[259, 9, dim - 32:] = want[299, 11, :32] = np.nan
    odd = np.isnan(want)
    assert np.array_equal(np.isnan(got), odd)
    attention_close(np.where(odd, 0, got), np.where(odd, 0, want), size, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale,q_scale", [(1e-3, 1.0), (0.5, 4.0), (8.0, 4.0)])
def test_attention_of_flat_and_sharp_scores(dtype, scale, q_scale):
    """With a large scale one key takes nearly all of a row's weight, and scores are in the hundreds; their error grows with them."""
    c = plain.Case(21, heads=4, kv_heads=2, dim=64, page=16, prefix=150, held=[70, 3], new=[2, 1], dtype=dtype, q_scale=q_scale)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, size = reference(c, K, V, 32, scale)
    # 2^-24 x 20 x sum |q k| scale (fp32 caches: 2^-23 more for a query's two fp16); sum |q k| is some 0.64 x 64 x q_scale
    extra = 2.0 ** -24 * (20 + 2) * 0.64 * 64 * q_scale * scale * 2
    attention_close(run_attention(c, K, V, 32, scale=scale), ref, size.max(), dtype, extra)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q_scale,size", [(2.0 ** -40, 1.0), (2.0 ** 40, 1.0), (1.0, 2.0 ** -16), (1.0, 2.0 ** 14)])
def test_attention_of_small_and_large_numbers(dtype, q_scale, size):
    """Queries of any size (with a scale that makes up for it); values whose fp16 are subnormal, which the format keeps to 2^-25, and as large as it holds."""
    check_attention(22, scale=0.125 / q_scale, size=size, heads=4, kv_heads=2, dim=128, page=16, prefix=70, held=[40, 3], new=[2, 1], dtype=dtype, q_scale=q_scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("new", [[1, 3], [70, 40]])
def test_attention_of_queries_that_are_zero_or_next_to_it(dtype, new):
    """rows without a largest feature, or with one below the normal numbers of fp32, weigh all their keys alike; their neighbours do not"""
    c = plain.Case(31, heads=8, kv_heads=4, dim=64, page=16, prefix=20, held=[300, 5], new=new, dtype=dtype)
    c.q[0], c.q[-1, 1], c.q[1, 2] = 0.0, -0.0, plain.stored(c.q[1, 2] * 2.0 ** -135, dtype)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, most = reference(c, K, V, 32, None)
    attention_close(run_attention(c, K, V, 32), ref, most, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_queries_with_one_large_feature(dtype):
    c = plain.Case(23, heads=4, kv_heads=2, dim=128, page=16, prefix=0, held=[60], new=[2], dtype=dtype)
    c.K[..., 7] *= 2.0 ** -12
    c.q[..., 7] = 4096.0
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, size = reference(c, K, V, 32, None)
    # the large feature's codes are one of its group's steps, so that products reach 4096 x 0.3: sums of |q k| scale of some 150
    attention_close(run_attention(c, K, V, 32), ref, size.max(), dtype, 2.0 ** -24 * 22 * 150 * 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,prefix", [(64, 0), (128, 0), (256, 0), (64, 300), (128, 20)])
def test_attention_keeps_what_later_tokens_hold_from_earlier_ones(dtype, dim, prefix):
    """Groups of NaN in the key or value of a new token reach the tokens that see it and no others; a group's features, and no others."""
    c = plain.Case(31, heads=4, kv_heads=2, dim=dim, page=16, prefix=prefix, held=[3, 30], new=[40, 9], dtype=dtype)
    at = lambda b, i: (c.pages[b, i // 16], i % 16)  # noqa: E731
    clean = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, size = reference(c, *clean, 32, None)
    K, V = (np.array(x) for x in clean)
    pairs_K, pairs_V = (q4_plain.parts(x, 2, dim, 16, 32)[1] for x in (K, V))
    nan = np.float16(np.nan), np.float16(0)

    def spoil(pool, page, head, slot, g):       # parts() may be a copy: the bytes themselves
        row, groups = q4_plain.sizes(dim, 32)
        block = pool.reshape(pool.shape[0], 2, -1)[page, head]
        block[16 * row:].view(np.float16).reshape(16, groups, 2)[slot, g] = nan

    spoil(K, *(lambda p, s: (p, 0, s))(*at(0, 3 + 25)), 1)       # kv head 0: scores not a number from the sequence's token 25 on
    spoil(V, *(lambda p, s: (p, 1, s))(*at(0, 3 + 10)), 0)
    spoil(V, *(lambda p, s: (p, 0, s))(*at(1, 30 + 8)), dim // 32 - 1)        # the last token's own
    got = run_attention(c, K, V, 32)
    want = ref.copy()
    want[25:40, 0:2] = np.nan
    want[10:40, 2:4, :32] = np.nan
    want[48, 0:2, dim - 32:] = np.nan
    odd = np.isnan(want)
    assert np.array_equal(np.isnan(got), odd)
    attention_close(np.where(odd, 0, got), np.where(odd, 0, want), size, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("fill", [0x00, 0x7B, 0x7C, 0xFC, 0xFF])
def test_attention_of_places_that_hold_anything(dtype, fill):
    """What lies behind a sequence's last token, and in the pages that its table does not use, is zeros, infinities, NaN and the largest numbers."""
    for held, new, prefix in (([0, 17, 40], [1, 1, 1], 5), ([0, 9], [40, 3], 0)):
        c = plain.Case(32, heads=4, kv_heads=2, dim=128, page=16, prefix=prefix, held=held, new=new, dtype=dtype)
        K, V = q4_plain.pool_of(c.K, 32, fill), q4_plain.pool_of(c.V, 32, fill)
        ref, size = reference(c, K, V, 32, None)
        attention_close(run_attention(c, K, V, 32), ref, size, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads,dim,prefix,held,new,max_len", [
    (4, 2, 64, 0, [5, 700, 0, 33], [1, 1, 1, 1], 4096),                  # far more room than is used
    (8, 1, 128, 0, [900, 0, 130, 129, 127], [3, 0, 5, 1, 4], 1000),      # several tiles of rows, a sequence without new tokens
    (8, 1, 128, 40, [900, 0, 130], [3, 2, 5], 2000),
    (4, 4, 64, 0, [3000], [1], 3001),
    (2, 2, 256, 10, [700, 3, 260], [1, 9, 20], 900),
    (20, 1, 64, 0, [300, 2, 513], [2, 3, 1], 600)])                      # tiles of 32 rows
def test_attention_of_parts_that_the_device_cuts(dtype, heads, kv_heads, dim, prefix, held, new, max_len):
    check_attention(19, heads=heads, kv_heads=kv_heads, dim=dim, page=16, prefix=prefix, held=held, new=new, dtype=dtype, max_len=max_len)


@pytest.mark.parametrize("n", [63, 64, 65, 200, 256])
def test_attention_of_many_sequences_that_the_device_cuts(n):
    rng = np.random.default_rng(n)
    check_attention(20, heads=2, kv_heads=1, dim=64, page=16, prefix=0, held=rng.integers(0, 400, n).tolist(), new=rng.integers(0, 3, n).tolist(), dtype=BF16, max_len=450)
    check_attention(20, heads=2, kv_heads=1, dim=64, page=16, prefix=30, held=rng.integers(0, 400, n).tolist(), new=[1] * n, dtype=BF16, max_len=450)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_beyond_max_len(dtype):
    check_attention(51, heads=4, kv_heads=2, dim=64, page=16, prefix=20, held=[60, 64, 100, 5], new=[8, 3, 1, 2], dtype=dtype, max_len=64)


def test_attention_of_a_group_of_infinite_queries_is_nan():
    c = plain.Case(41, heads=2, kv_heads=1, dim=64, page=16, prefix=0, held=[4], new=[2], dtype=BF16)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, size = reference(c, K, V, 32, None)
    c.q[0, 1, 9] = np.nan
    c.q[1, 0, 3], c.q[1, 0, 4] = np.inf, -np.inf
    got = run_attention(c, K, V, 32)
    bad = np.zeros((2, 2), bool)
    bad[0, 1] = bad[1, 0] = True
    assert np.array_equal(np.isnan(got).all(axis=2), bad) and np.array_equal(np.isnan(got).any(axis=2), bad)
    attention_close(got[~bad], ref[~bad], size[~bad], BF16)


def test_attention_offsets_past_32_bits():
    """Pools of 5 GB each, the pages in use at their ends."""
    heads, dim, page = 8, 128, 256
    size = G.griffin_kv_q4_page_bytes(heads, dim, page)
    n = (5 << 30) // size
    c = plain.Case(61, heads=heads, kv_heads=heads, dim=dim, page=page, prefix=300, held=[5, 250], new=[2, 9], dtype=BF16)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, most = reference(c, K, V, 32, None)
    pools = []
    for x in (K, V):
        pool = torch.empty(n, size, dtype=torch.uint8, device="cuda")
        pool[n - c.n_pages:] = put(x)
        pools.append(pool)
    shift = n - c.n_pages
    C = cache(c, *pools, 32)
    B = G.kv_batch(c.cu, ints(c.lens), ints(c.pages + shift), c.max_len, prefix_pages=ints(c.prefix_pages + shift), n_prefix=c.prefix)
    q, out = dev(c.q, BF16), torch.zeros(c.q.shape, dtype=torch.bfloat16, device="cuda")
    G.griffin_attention_q4(C, B, q, out, workspace=workspace(G.griffin_attention_q4_workspace_bytes(C, B, heads)))
    attention_close(to_host(out), ref, most, BF16)
    k, v = dev(c.k, BF16), dev(c.v, BF16)
    G.griffin_kv_append_q4(C, B, k, v)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    G.griffin_kv_read_q4(C, B, k2, v2)
    codes, pairs = q4_plain.pack(c.k, 32)
    assert torch.equal(k2, dev(q4_plain.values(codes, pairs, dim, 32), BF16))


def test_results_do_not_depend_on_the_run():
    c = plain.Case(71, heads=32, kv_heads=8, dim=128, page=64, prefix=3000, held=[0, 150, 7], new=[1, 5, 2], dtype=BF16)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    first = run_attention(c, K, V, 32)
    for _ in range(3):
        assert np.array_equal(run_attention(c, K, V, 32), first)


def test_step_on_another_stream_and_in_a_graph():
    """A step's calls captured once and replayed with other tokens and lengths, eager work between; every replay is the eager call's bit for bit."""
    c = plain.Case(81, heads=8, kv_heads=2, dim=128, page=16, prefix=40, held=[3, 20], new=[2, 2], dtype=BF16, max_len=64)
    c.pages = np.arange(c.pages.size, dtype=np.int32).reshape(c.pages.shape) + 3
    n = 3 + c.pages.size
    c.prefix_pages = np.arange(3, dtype=np.int32)
    rng = np.random.default_rng(1)
    x = [q4_plain.pool_of(plain.stored(rng.standard_normal((n, 2, 16, 128)), BF16), 32) for _ in range(2)]
    stream = torch.cuda.Stream()
    lens, pages, prefix_pages = ints(c.lens), ints(c.pages), ints(c.prefix_pages)
    B = G.kv_batch(c.cu, lens, pages, c.max_len, prefix_pages=prefix_pages, n_prefix=c.prefix)
    q, k, v = (dev(a, BF16) for a in (c.q, c.k, c.v))
    cos, sin = (torch.from_numpy(np.asarray(t, np.float32)).cuda() for t in tables(c.prefix + c.max_len, 128))

    def setup():
        K, V = put(x[0]), put(x[1])
        C = cache(c, K, V, 32)
        return dict(C=C, K=K, V=V, q_out=torch.zeros_like(q), out=torch.zeros_like(q), ws=workspace(G.griffin_attention_q4_workspace_bytes(C, B, 8)),
                    k2=torch.zeros_like(k), v2=torch.zeros_like(v))

    def step(s):
        G.griffin_kv_append_q4(s["C"], B, k, v, q=q, q_out=s["q_out"], cos=cos, sin=sin)
        G.griffin_attention_q4(s["C"], B, s["q_out"], s["out"], workspace=s["ws"])
        G.griffin_kv_read_q4(s["C"], B, s["k2"], s["v2"])

    a, b = setup(), setup()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step(a)
    stream.synchronize()
    a = setup()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step(a)
    for i in range(4):
        lens.add_(2)
        for t in (q, k, v):
            t.copy_(t.flip(0) * (0.5 + i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(b)
        torch.cuda.synchronize()
        for name in ("K", "V", "q_out", "out", "k2", "v2"):
            assert torch.equal(a[name], b[name]), (i, name)


def test_graphs_that_share_a_workspace():
    """Two batches' calls captured into graphs with one workspace, replayed in turn on one stream"""
    cases, graphs = [], []
    ws = None
    for seed, held, new, prefix in ((91, [5, 700, 33], [1, 1, 1], 0), (92, [3, 90], [4, 70], 300)):
        c = plain.Case(seed, heads=8, kv_heads=2, dim=128, page=16, prefix=prefix, held=held, new=new, dtype=BF16)
        K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
        cases.append((cache(c, put(K), put(V), 32), batch(c), dev(c.q, BF16), torch.zeros(c.q.shape, dtype=torch.bfloat16, device="cuda"), *reference(c, K, V, 32, None)))
    ws = workspace(max(G.griffin_attention_q4_workspace_bytes(C, B, 8) for C, B, *_ in cases))
    stream = torch.cuda.Stream()
    for C, B, q, out, *_ in cases:
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            G.griffin_attention_q4(C, B, q, out, workspace=ws)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            G.griffin_attention_q4(C, B, q, out, workspace=ws)
        graphs.append(graph)
    for _ in range(3):
        for _, _, _, out, *_ in cases:
            out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for graph in graphs:
                graph.replay()
        stream.synchronize()
        for _, _, _, out, ref, size in cases:
            attention_close(to_host(out), ref, size, BF16)


def test_append_of_more_workgroups_than_one_launch_takes():
    """2^20 tokens of 17 workgroups each: the step goes out in parts, and its first and last tokens are what a small step makes of them"""
    heads, dim, n, page = 544, 8, 1 << 20, 65536
    size = G.griffin_kv_q4_page_bytes(heads, dim, page)
    K, V = (torch.zeros(n // page, size, dtype=torch.uint8, device="cuda") for _ in range(2))
    C = G.kv_cache_q4(K, V, kv_heads=heads, dim=dim, page_size=page, dtype=torch.bfloat16)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    k, v = (torch.empty(n, heads, dim, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    pages = ints([list(range(n // page))])
    G.griffin_kv_append_q4(C, G.kv_batch([0, n], ints([0]), pages, n), k, v)
    most = ((1 << 24) - 1) // 17                 # tokens of the first part
    for at in (0, most - 8, n - 16):
        back = [torch.zeros(16, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        G.griffin_kv_read_q4(C, G.kv_batch([0, 16], ints([at]), pages, n), *back)
        for x, y in zip((k, v), back):
            codes, pairs = q4_plain.pack(to_host(x[at:at + 16]), 32)
            assert torch.equal(y, dev(q4_plain.values(codes, pairs, dim, 32), BF16))
