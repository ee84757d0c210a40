"""Host-side checks of the cache in 4 bits and of the verification of drafted tokens, without a GPU: layouts, sizes, refusals before any HIP call."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2404_01365_amd as G
import q4_plain
from test_layer_abi_cpu import FAKE, mk_batch

lib, ref = G.lib, ctypes.byref


def test_struct_layout_matches_header():
    assert ctypes.sizeof(G.griffin_kv_cache_q4) == 48
    assert [getattr(G.griffin_kv_cache_q4, f).offset for f in ("V", "dtype", "dim", "group", "n_pages")] == [8, 16, 24, 32, 40]


@pytest.mark.parametrize("kv_heads,dim,page,group", [(8, 128, 16, 32), (1, 8, 16, 64), (5, 80, 64, 32), (3, 96, 32, 64), (2, 256, 65536, 32), (1024, 40, 16, 32)])
def test_page_bytes(kv_heads, dim, page, group):
    assert G.griffin_kv_q4_page_bytes(kv_heads, dim, page, group) == q4_plain.page_bytes(kv_heads, dim, page, group)


@pytest.mark.parametrize("bad", [(0, 128, 16, 32), (1025, 128, 16, 32), (8, 0, 16, 32), (8, 12, 16, 32), (8, 264, 16, 32), (8, 128, 8, 32), (8, 128, 24, 32),
                                 (8, 128, 131072, 32), (8, 128, 16, 16), (8, 128, 16, 128), (-1, 128, 16, 32)])
def test_page_bytes_of_what_is_refused(bad):
    assert G.griffin_kv_q4_page_bytes(*bad) == 0


def mk_cache(**kw):
    C = G.griffin_kv_cache_q4()
    C.K, C.V, C.dtype, C.kv_heads, C.dim, C.page_size, C.group, C.n_pages = FAKE, FAKE, G.BF16, 8, 128, 16, 32, 100
    for k, v in kw.items():
        setattr(C, k, v)
    return C


def append(C, B, k=FAKE, ldk=1024, hsk=128, v=FAKE, ldv=1024, hsv=128, q=FAKE, ldq=4096, hsq=128, q_out=FAKE, ldo=4096, hso=128, heads=32,
           cos=FAKE, sin=FAKE, n_pos=1000, rot=128, style=0):
    return lib.griffin_kv_append_q4(None if C is None else ref(C), None if B is None else ref(B), k, ldk, hsk, v, ldv, hsv, q, ldq, hsq, q_out, ldo, hso, heads,
                                    cos, sin, n_pos, rot, style, None)


def read(C, B, k=FAKE, ldk=1024, hsk=128, v=FAKE + 4096, ldv=1024, hsv=128):
    return lib.griffin_kv_read_q4(None if C is None else ref(C), None if B is None else ref(B), k, ldk, hsk, v, ldv, hsv, None)


def attend(C, B, q=FAKE, ldq=4096, hsq=128, out=FAKE + 4096, ldo=4096, hso=128, heads=32, scale=0.1, ws=FAKE, size=1 << 30):
    return lib.griffin_attention_q4(None if C is None else ref(C), None if B is None else ref(B), q, ldq, hsq, out, ldo, hso, heads, scale, ws, size, None)


CACHES = [(G.EINVAL, dict(K=None)), (G.EINVAL, dict(V=None)), (G.EINVAL, dict(dtype=2)), (G.EINVAL, dict(kv_heads=0)), (G.EINVAL, dict(dim=0)), (G.EINVAL, dict(page_size=0)),
          (G.EINVAL, dict(group=0)), (G.EINVAL, dict(n_pages=0)), (G.ESHAPE, dict(dim=124)), (G.ESHAPE, dict(K=FAKE + 8)), (G.ESHAPE, dict(V=FAKE + 4)),
          (G.ESHAPE, dict(n_pages=1 << 31)), (G.EUNSUPPORTED, dict(dim=264)), (G.EUNSUPPORTED, dict(page_size=8)), (G.EUNSUPPORTED, dict(page_size=48)),
          (G.EUNSUPPORTED, dict(page_size=131072)), (G.EUNSUPPORTED, dict(group=16)), (G.EUNSUPPORTED, dict(group=128)), (G.EUNSUPPORTED, dict(kv_heads=1025))]
BATCHES = [(G.EINVAL, dict(cu_seqlens=None)), (G.EINVAL, dict(n_seqs=0)), (G.EINVAL, dict(max_len=0)), (G.EINVAL, dict(lens=None)), (G.EINVAL, dict(pages=None)),
           (G.EINVAL, dict(n_prefix=-1)), (G.EINVAL, dict(prefix_pages=None)), (G.EUNSUPPORTED, dict(n_seqs=257)), (G.ESHAPE, dict(ld_pages=3)),
           (G.ESHAPE, dict(max_len=1 << 30, ld_pages=1 << 27))]


@pytest.mark.parametrize("call", [append, read, attend])
@pytest.mark.parametrize("status,kw", CACHES)
def test_caches_that_are_refused(call, status, kw):
    assert call(mk_cache(**kw), mk_batch()) == status
    assert lib.griffin_attention_q4_workspace_bytes(ref(mk_cache(**kw)), ref(mk_batch()), 32) == 0


@pytest.mark.parametrize("call", [append, read, attend])
@pytest.mark.parametrize("status,kw", BATCHES)
def test_batches_that_are_refused(call, status, kw):
    assert call(mk_cache(), mk_batch(**kw)) == status


@pytest.mark.parametrize("call", [append, read, attend])
def test_what_else_is_refused_and_what_is_nothing_to_do(call):
    assert call(None, mk_batch()) == G.EINVAL and call(mk_cache(), None) == G.EINVAL
    assert call(mk_cache(), mk_batch((1, 2))) == G.ESHAPE and call(mk_cache(), mk_batch((0, 3, 2))) == G.ESHAPE
    assert call(mk_cache(), mk_batch((0, (1 << 20) + 1))) == G.EUNSUPPORTED
    assert call(mk_cache(), mk_batch((0, 0, 0))) == G.OK


@pytest.mark.parametrize("status,kw", [
    (G.EINVAL, dict(k=None)), (G.EINVAL, dict(v=None)), (G.EINVAL, dict(q=None)), (G.EINVAL, dict(q_out=None)), (G.EINVAL, dict(rot=-2)), (G.EINVAL, dict(cos=None)),
    (G.EINVAL, dict(n_pos=0)), (G.EINVAL, dict(style=2)), (G.EINVAL, dict(heads=0)), (G.ESHAPE, dict(rot=130)), (G.ESHAPE, dict(rot=7)), (G.ESHAPE, dict(ldk=100)),
    (G.ESHAPE, dict(hsv=12)), (G.ESHAPE, dict(k=FAKE + 8)), (G.ESHAPE, dict(ldq=4092)), (G.ESHAPE, dict(hso=64)), (G.ESHAPE, dict(ldo=4104)), (G.ESHAPE, dict(cos=FAKE + 4)),
    (G.EUNSUPPORTED, dict(heads=1025))])
def test_append_refuses(status, kw):
    assert append(mk_cache(), mk_batch(), **kw) == status


@pytest.mark.parametrize("status,kw", [(G.EINVAL, dict(k=None, v=None)), (G.EINVAL, dict(k=FAKE, v=FAKE)), (G.ESHAPE, dict(ldk=120)), (G.ESHAPE, dict(hsv=132)),
                                       (G.ESHAPE, dict(v=FAKE + 8)), (G.ESHAPE, dict(k=FAKE + 2))])
def test_read_refuses(status, kw):
    assert read(mk_cache(), mk_batch(), **kw) == status


@pytest.mark.parametrize("status,kw", [
    (G.EINVAL, dict(q=None)), (G.EINVAL, dict(out=None)), (G.EINVAL, dict(out=FAKE)), (G.EINVAL, dict(scale=0.0)), (G.EINVAL, dict(scale=float("nan"))),
    (G.EINVAL, dict(scale=float("inf"))), (G.EINVAL, dict(heads=0)), (G.ESHAPE, dict(heads=33)), (G.EUNSUPPORTED, dict(heads=1032)), (G.ESHAPE, dict(ldq=4100)),
    (G.ESHAPE, dict(hso=64)), (G.ESHAPE, dict(q=FAKE + 8)), (G.EWORKSPACE, dict(ws=None)), (G.EWORKSPACE, dict(ws=FAKE + 128)), (G.EWORKSPACE, dict(size=16))])
def test_attention_refuses(status, kw):
    C, B = mk_cache(), mk_batch(n_prefix=5000)
    assert lib.griffin_attention_q4_workspace_bytes(ref(C), ref(B), 32) > 16
    assert attend(C, B, **kw) == status


def test_attention_refuses_more_rows_than_it_counts():
    B = mk_batch((0, 1 << 20))
    assert lib.griffin_attention_q4_workspace_bytes(ref(mk_cache()), ref(B), 32) == 0
    assert attend(mk_cache(), B) == G.EUNSUPPORTED


def test_workspace_goes_by_sizes_alone():
    C, B = mk_cache(), mk_batch(n_prefix=5000)
    want = lib.griffin_attention_q4_workspace_bytes(ref(C), ref(B), 32)
    assert lib.griffin_attention_q4_workspace_bytes(ref(C), ref(mk_batch(n_prefix=5000, lens=None, pages=None, prefix_pages=None, ld_pages=0)), 32) == want


# ----------------------------------------------------------------------------------------------- drafted tokens
def verify(cu=(0, 5, 9), n_seqs=None, vocab=1000, p=FAKE, ldp=1000, q=FAKE, ldq=1000, drafted=FAKE, u=FAKE, r=FAKE, tokens=FAKE + 4096, accepted=FAKE, lens=FAKE,
           lens_out=FAKE, ws=FAKE, size=1 << 20):
    arr = None if cu is None else (ctypes.c_int32 * len(cu))(*cu)
    return lib.griffin_verify_drafts(p, ldp, q, ldq, drafted, arr, len(cu) - 1 if n_seqs is None else n_seqs, vocab, u, r, tokens, accepted, lens, lens_out, ws, size, None)


@pytest.mark.parametrize("status,kw", [
    (G.EINVAL, dict(cu=None, n_seqs=2)), (G.EINVAL, dict(n_seqs=0)), (G.EINVAL, dict(vocab=0)), (G.EINVAL, dict(p=None)), (G.EINVAL, dict(drafted=None)),
    (G.EINVAL, dict(u=None)), (G.EINVAL, dict(r=None)), (G.EINVAL, dict(tokens=None)), (G.EINVAL, dict(accepted=None)), (G.EINVAL, dict(tokens=FAKE)),
    (G.EINVAL, dict(lens=None)), (G.EINVAL, dict(lens_out=None)), (G.EUNSUPPORTED, dict(vocab=(1 << 24) + 1, ldp=1 << 25, ldq=1 << 25)),
    (G.EUNSUPPORTED, dict(cu=range(258))), (G.ESHAPE, dict(cu=(1, 2))), (G.ESHAPE, dict(cu=(0, 3, 2))), (G.ESHAPE, dict(ldp=999)), (G.ESHAPE, dict(ldq=10)),
    (G.ESHAPE, dict(p=FAKE + 2)), (G.ESHAPE, dict(lens_out=FAKE + 1)), (G.EWORKSPACE, dict(ws=FAKE + 64)), (G.EWORKSPACE, dict(vocab=100000, ldp=100000, ldq=100000, size=8)),
    (G.EWORKSPACE, dict(vocab=100000, ldp=100000, ldq=100000, ws=None))])
def test_verify_refuses(status, kw):
    if kw.get("ws") == FAKE + 64:
        kw = dict(kw, vocab=100000, ldp=100000, ldq=100000)
    assert verify(**kw) == status


def test_verify_workspace_of_what_is_refused():
    for n, vocab in ((0, 100), (257, 100), (1, 0), (1, (1 << 24) + 1), (-1, 5)):
        assert G.griffin_verify_workspace_bytes(n, vocab) == 0


# ----------------------------------------------------------------------------------------------- the binding
def test_binding_refuses_pools_that_do_not_fit():
    size = G.griffin_kv_q4_page_bytes(2, 64, 16)
    K = torch.zeros(3, size, dtype=torch.uint8)
    kw = dict(kv_heads=2, dim=64, page_size=16, dtype=torch.bfloat16)
    G.kv_cache_q4(K, K.clone(), **kw)
    for bad in (K[:, :-16], K[:2], K.view(torch.int8), torch.zeros(3, size + 16, dtype=torch.uint8)[:, :size]):
        with pytest.raises((ValueError, TypeError)):
            G.kv_cache_q4(K, bad, **kw)
    with pytest.raises(ValueError):
        G.kv_cache_q4(K, K, kv_heads=2, dim=64, page_size=16, group=48, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        G.kv_cache_q4(K, K, kv_heads=2, dim=64, page_size=16, dtype=torch.float16)


def test_binding_refuses_tensors_on_the_host():
    size = G.griffin_kv_q4_page_bytes(2, 64, 16)
    K, V = torch.zeros(3, size, dtype=torch.uint8), torch.zeros(3, size, dtype=torch.uint8)
    C = G.kv_cache_q4(K, V, kv_heads=2, dim=64, page_size=16, dtype=torch.float32)
    B = G.kv_batch([0, 1], torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), 4)
    k, v = torch.zeros(1, 2, 64), torch.zeros(1, 2, 64)
    for call in (lambda: G.griffin_kv_append_q4(C, B, k, v), lambda: G.griffin_kv_read_q4(C, B, k, v), lambda: G.griffin_attention_q4(C, B, k, v)):
        with pytest.raises(ValueError, match="host"):
            call()
    p = torch.full((2, 10), 0.1)
    i, f = torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(ValueError, match="host"):
        G.griffin_verify_drafts([0, 2], p, i, f, f[:1], i.clone(), i[:1].clone())
    for kw in (dict(p=p.double()), dict(drafted=i.long()), dict(accept_u=f[:1]), dict(draw_u=f), dict(tokens_out=i[:1]), dict(accepted=i), dict(draft_p=p[:1])):
        args = dict(p=p, drafted=i, accept_u=f, draw_u=f[:1], tokens_out=i.clone(), accepted=i[:1].clone())
        args.update(kw)
        with pytest.raises((ValueError, TypeError)):
            G.griffin_verify_drafts([0, 2], **args)


# ----------------------------------------------------------------------------------------------- the definitions themselves
@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("dim", [8, 40, 96, 128])
def test_values_come_back_within_half_a_step(dim, group):
    rng = np.random.default_rng(dim + group)
    x = rng.standard_normal((50, dim)) * 10.0 ** rng.uniform(-2, 3, (50, 1)) + rng.standard_normal((50, 1)) * 5
    codes, pairs = q4_plain.pack(x, group)
    back = q4_plain.values(codes, pairs, dim, group)
    f = np.arange(dim) // group
    step, most = pairs[..., 0].astype(np.float64)[:, f], np.stack([np.abs(x[:, f == g]).max(axis=1) for g in range(f[-1] + 1)], axis=1)[:, f]
    # half a step, and what fp16 takes from the scale (15 steps of it), the middle and the value
    assert np.all(np.abs(back - x) <= step / 2 + 2.0 ** -11 * (most + 8 * step) + 2.0 ** -24)
