"""Host-side checks of what surrounds the FF block, without a GPU: layouts of the descriptors, refusals before any HIP call, workspaces."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import paper_2404_01365_amd as G
from test_launch_errors import SHIM

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000001000          # never dereferenced on these paths (256-byte aligned)
lib, ref = G.lib, ctypes.byref


def test_struct_layouts_match_header():
    assert ctypes.sizeof(G.griffin_norm) == 64 and G.griffin_norm.w_pre.offset == 32
    assert ctypes.sizeof(G.griffin_kv_cache) == 64 and G.griffin_kv_cache.n_pages.offset == 32
    assert ctypes.sizeof(G.griffin_kv_batch) == 56 and G.griffin_kv_batch.lens.offset == 16 and G.griffin_kv_batch.prefix_pages.offset == 48


def mk_norm(**kw):
    N = G.griffin_norm()
    N.d, N.dtype, N.kind, N.eps, N.h_scale, N.y_scale, N.w_pre = 512, G.BF16, G.NORM_RMS, 1e-5, 1.0, 1.0, FAKE
    for k, v in kw.items():
        setattr(N, k, v)
    return N


def call_norm(N, rows=4, h=FAKE, ldh=512, h_dtype=G.BF16, y=FAKE, ldy=512, gate=None, ldg=0, h_out=FAKE, ldo=512, x=FAKE + 4096, ldx=512):
    return lib.griffin_norm_residual(ref(N) if N is not None else None, rows, h, ldh, h_dtype, y, ldy, gate, ldg, h_out, ldo, x, ldx, None)


@pytest.mark.parametrize("status,norm_kw,kw", [
    (G.EINVAL, dict(d=0), {}), (G.EINVAL, dict(d=-8), {}), (G.EINVAL, dict(dtype=2), {}), (G.EINVAL, dict(kind=2), {}),
    (G.EINVAL, dict(eps=0.0), {}), (G.EINVAL, dict(eps=float("nan")), {}), (G.EINVAL, dict(eps=float("inf")), {}),
    (G.EINVAL, dict(h_scale=float("inf")), {}), (G.EINVAL, dict(y_scale=float("nan")), {}), (G.EINVAL, dict(w_offset=float("nan")), {}),
    (G.EINVAL, dict(w_pre=None), {}), (G.EINVAL, dict(w_pre=None, b_pre=FAKE), dict(x=None)), (G.EINVAL, dict(b_post=FAKE), {}),
    (G.EINVAL, {}, dict(rows=-1)), (G.EINVAL, {}, dict(h=None)), (G.EINVAL, {}, dict(h_out=None, x=None)), (G.EINVAL, {}, dict(h_dtype=5)),
    (G.EINVAL, {}, dict(y=None, gate=FAKE)),
    (G.ESHAPE, dict(d=516), dict(ldh=520, ldy=520, ldo=520, ldx=520)), (G.ESHAPE, {}, dict(ldh=504)), (G.ESHAPE, {}, dict(ldy=516)),
    (G.ESHAPE, {}, dict(gate=FAKE, ldg=504)), (G.ESHAPE, {}, dict(ldx=0)), (G.ESHAPE, {}, dict(h=FAKE + 8, h_out=None)),
    (G.ESHAPE, {}, dict(x=FAKE + 2)), (G.ESHAPE, dict(w_post=FAKE + 4), {}), (G.ESHAPE, {}, dict(ldo=520)),        # in place with another stride
    (G.ESHAPE, {}, dict(x=FAKE, h_out=None, ldx=520)), (G.EINVAL, {}, dict(x=FAKE)), (G.ESHAPE, {}, dict(rows=2 ** 30 + 1)),
    (G.EUNSUPPORTED, dict(d=32776), dict(ldh=32776, ldy=32776, ldo=32776, ldx=32776)),
    (G.EUNSUPPORTED, dict(dtype=G.F32), {}),                     # a bf16 stream beside fp32 blocks
    (G.OK, {}, dict(rows=0, h=None, x=None, h_out=None)),
])
def test_norm_refuses(status, norm_kw, kw):
    assert call_norm(mk_norm(**norm_kw), **kw) == status


def test_norm_refuses_no_descriptor():
    assert call_norm(None) == G.EINVAL


def mk_cache(**kw):
    C = G.griffin_kv_cache()
    C.K, C.V, C.dtype, C.kv_heads, C.dim, C.page_size, C.n_pages = FAKE, FAKE, G.BF16, 8, 128, 16, 100
    C.page_stride, C.head_stride, C.token_stride = 8 * 16 * 128, 16 * 128, 128
    for k, v in kw.items():
        setattr(C, k, v)
    return C


def mk_batch(cu=(0, 1, 2), **kw):
    B = G.griffin_kv_batch()
    arr = (ctypes.c_int32 * len(cu))(*cu)
    B._arr = arr
    B.cu_seqlens, B.n_seqs, B.max_len = ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32)), len(cu) - 1, 64
    B.lens, B.pages, B.ld_pages, B.n_prefix, B.prefix_pages = FAKE, FAKE, 4, 100, FAKE
    for k, v in kw.items():
        setattr(B, k, v)
    return B


def append(C, B, k=FAKE, ldk=1024, hsk=128, v=FAKE, ldv=1024, hsv=128, q=FAKE, ldq=4096, hsq=128, q_out=FAKE, ldo=4096, hso=128, heads=32,
           cos=FAKE, sin=FAKE, n_pos=1000, rot=128, style=0):
    return lib.griffin_kv_append(ref(C), ref(B), k, ldk, hsk, v, ldv, hsv, q, ldq, hsq, q_out, ldo, hso, heads, cos, sin, n_pos, rot, style, None)


def attend(C, B, q=FAKE, ldq=4096, hsq=128, out=FAKE + 4096, ldo=4096, hso=128, heads=32, scale=0.1, ws=FAKE, ws_bytes=1 << 40):
    return lib.griffin_attention(ref(C), ref(B), q, ldq, hsq, out, ldo, hso, heads, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("status,cache_kw,batch_kw", [
    (G.EINVAL, dict(K=None), {}), (G.EINVAL, dict(V=None), {}), (G.EINVAL, dict(dtype=3), {}), (G.EINVAL, dict(kv_heads=0), {}),
    (G.EINVAL, dict(dim=0), {}), (G.EINVAL, dict(page_size=0), {}), (G.EINVAL, dict(n_pages=0), {}),
    (G.ESHAPE, dict(dim=124), {}), (G.ESHAPE, dict(K=FAKE + 8), {}), (G.ESHAPE, dict(token_stride=120), {}), (G.ESHAPE, dict(token_stride=132), {}),
    (G.ESHAPE, dict(head_stride=64), {}), (G.ESHAPE, dict(page_stride=-8), {}), (G.ESHAPE, dict(page_stride=12), {}),
    (G.ESHAPE, dict(n_pages=2 ** 31), {}),
    (G.EUNSUPPORTED, dict(dim=264, token_stride=264, head_stride=264), {}), (G.EUNSUPPORTED, dict(page_size=8), {}),
    (G.EUNSUPPORTED, dict(page_size=48), {}), (G.EUNSUPPORTED, dict(page_size=2 ** 17), {}), (G.EUNSUPPORTED, dict(kv_heads=1025), {}),
    (G.EINVAL, {}, dict(cu_seqlens=None)), (G.EINVAL, {}, dict(n_seqs=0)), (G.EINVAL, {}, dict(max_len=0)), (G.EINVAL, {}, dict(n_prefix=-1)),
    (G.EINVAL, {}, dict(lens=None)), (G.EINVAL, {}, dict(pages=None)), (G.EINVAL, {}, dict(prefix_pages=None)),
    (G.ESHAPE, {}, dict(ld_pages=3)), (G.ESHAPE, {}, dict(cu=(1, 2))), (G.ESHAPE, {}, dict(cu=(0, 3, 2))),
    (G.ESHAPE, {}, dict(max_len=2 ** 30 + 1, ld_pages=2 ** 40)), (G.ESHAPE, {}, dict(n_prefix=2 ** 30 + 1)), (G.ESHAPE, {}, dict(n_prefix=2 ** 30 - 63)),
    (G.EUNSUPPORTED, {}, dict(cu=tuple(range(G.MAX_SEQS + 2)))), (G.EUNSUPPORTED, {}, dict(cu=(0, 2 ** 20 + 1))),
    (G.OK, {}, dict(cu=(0, 0, 0))),
])
def test_cache_and_batch_are_checked(status, cache_kw, batch_kw):
    C, B = mk_cache(**cache_kw), mk_batch(**batch_kw)
    assert append(C, B) == status and attend(C, B) == status
    sizes = status == G.OK or any(k in batch_kw for k in ("lens", "pages", "prefix_pages", "ld_pages")) and len(batch_kw) == 1
    assert sizes or G.griffin_attention_workspace_bytes(C, B, 32) == 0
    assert lib.griffin_kv_append(None, ref(B), *([FAKE, 1024, 128] * 4), 32, FAKE, FAKE, 10, 0, 0, None) == G.EINVAL
    assert lib.griffin_attention(ref(mk_cache()), None, FAKE, 4096, 128, FAKE + 64, 4096, 128, 32, 1.0, FAKE, 1 << 40, None) == G.EINVAL


@pytest.mark.parametrize("status,kw", [
    (G.EINVAL, dict(k=None)), (G.EINVAL, dict(v=None)), (G.EINVAL, dict(q=None)), (G.EINVAL, dict(q_out=None)), (G.EINVAL, dict(rot=-2)),
    (G.EINVAL, dict(cos=None)), (G.EINVAL, dict(sin=None)), (G.EINVAL, dict(n_pos=0)), (G.EINVAL, dict(heads=0)), (G.EINVAL, dict(style=2)),
    (G.ESHAPE, dict(rot=130)), (G.ESHAPE, dict(rot=63)), (G.ESHAPE, dict(ldk=64)), (G.ESHAPE, dict(hsk=132)), (G.ESHAPE, dict(hsv=64)),
    (G.ESHAPE, dict(ldv=1028)), (G.ESHAPE, dict(k=FAKE + 2)), (G.ESHAPE, dict(q=FAKE + 8)), (G.ESHAPE, dict(cos=FAKE + 4)), (G.ESHAPE, dict(hsq=120)),
    (G.ESHAPE, dict(ldo=4100)), (G.ESHAPE, dict(ldo=8192)),                     # in place with another stride
    (G.EUNSUPPORTED, dict(heads=1025)),
])
def test_append_refuses(status, kw):
    assert append(mk_cache(), mk_batch(), **kw) == status


@pytest.mark.parametrize("status,kw", [
    (G.EINVAL, dict(q=None)), (G.EINVAL, dict(out=None)), (G.EINVAL, dict(out=FAKE)), (G.EINVAL, dict(scale=0.0)), (G.EINVAL, dict(scale=-1.0)),
    (G.EINVAL, dict(scale=float("nan"))), (G.EINVAL, dict(scale=float("inf"))), (G.EINVAL, dict(heads=0)),
    (G.ESHAPE, dict(heads=30)), (G.ESHAPE, dict(ldq=64)), (G.ESHAPE, dict(hsq=132)), (G.ESHAPE, dict(out=FAKE + 8)), (G.ESHAPE, dict(hso=0)),
    (G.EUNSUPPORTED, dict(heads=1032)),
    (G.EWORKSPACE, dict(ws=None)), (G.EWORKSPACE, dict(ws=FAKE + 16)), (G.EWORKSPACE, dict(ws_bytes=64)),
])
def test_attention_refuses(status, kw):
    assert attend(mk_cache(), mk_batch(n_prefix=2000), **kw) == status


def test_attention_workspace_is_enough_and_needed():
    C, B = mk_cache(), mk_batch(n_prefix=2000)
    need = G.griffin_attention_workspace_bytes(C, B, 32)
    assert need > 0 and attend(C, B, ws_bytes=need - 1) == G.EWORKSPACE
    assert G.griffin_attention_workspace_bytes(C, B, 30) == 0 and G.griffin_attention_workspace_bytes(C, B, 1032) == 0
    # device pointers and strides do not enter
    assert G.griffin_attention_workspace_bytes(C, mk_batch(n_prefix=2000, lens=None, pages=None, prefix_pages=None, ld_pages=0), 32) == need
    # one chunk of keys and nothing shared: written at once
    assert G.griffin_attention_workspace_bytes(mk_cache(), mk_batch(n_prefix=0, max_len=1), 32) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    t = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    with pytest.raises(TypeError):
        G.norm(t(64).double(), eps=1e-5)
    with pytest.raises(ValueError):
        G.norm(t(64), b_pre=t(32), eps=1e-5)
    with pytest.raises(TypeError):
        G.norm(t(64), w_post=t(64, dtype=torch.bfloat16), eps=1e-5)
    N = G.norm(t(64), eps=1e-5)
    for bad in (dict(y=t(3, 64)), dict(y=t(2, 32)), dict(y=t(64, 2).t()), dict(x=t(2, 64)[:1]), dict(gate=t(3, 64)), dict(gate=t(32))):
        with pytest.raises(ValueError):
            G.griffin_norm_residual(N, t(2, 64), bad.pop("y", t(2, 64)), t(2, 64), bad.pop("x", t(2, 64)), stream=1, **bad)
    with pytest.raises(TypeError):
        G.griffin_norm_residual(N, t(2, 64), t(2, 64, dtype=torch.bfloat16), t(2, 64), t(2, 64), stream=1)
    K = t(9, 2, 16, 64)
    with pytest.raises(ValueError):
        G.kv_cache(K, t(9, 16, 2, 64).transpose(1, 2))
    with pytest.raises(ValueError):
        G.kv_cache(K, t(9, 2, 16, 32))
    with pytest.raises(TypeError):
        G.kv_cache(K, K.bfloat16())
    C = G.kv_cache(K, K)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(TypeError):
        G.kv_batch([0, 1], i(1).long(), i(1, 2), 20)
    with pytest.raises(ValueError):
        G.kv_batch([0, 1], i(2), i(1, 2), 20)
    with pytest.raises(ValueError):
        G.kv_batch([0, 1, 2], i(2), i(1, 2).expand(2, 2), 20)
    good = dict(k=t(1, 2, 64), v=t(1, 2, 64), stream=1)
    with pytest.raises(ValueError):                              # 33 tokens in two pages of 16
        G.griffin_kv_append(C, G.kv_batch([0, 1], i(1), i(1, 2), 33), **good)
    with pytest.raises(ValueError):
        G.griffin_attention(C, G.kv_batch([0, 1], i(1), i(1, 2), 20, prefix_pages=i(1), n_prefix=17), t(1, 4, 64), t(1, 4, 64), stream=1)
    B = G.kv_batch([0, 1], i(1), i(1, 2), 20)
    for bad in (dict(k=t(2, 2, 64)), dict(v=t(1, 2, 32)), dict(q=t(1, 4, 64), q_out=t(1, 2, 64)), dict(cos=t(30, 32), sin=t(30, 16)),
                dict(cos=t(32, 30).t(), sin=t(32, 30).t())):
        with pytest.raises(ValueError):
            G.griffin_kv_append(C, B, **dict(good, **bad))
    with pytest.raises(TypeError):
        G.griffin_attention(C, B, t(1, 4, 64).bfloat16(), t(1, 4, 64), stream=1)
    with pytest.raises(ValueError):
        G.griffin_attention(C, B, t(1, 4, 64), t(2, 4, 64), stream=1)


CALLS = """
import ctypes, sys
shim = ctypes.CDLL(sys.argv[1])
sys.path.insert(0, sys.argv[2])
import paper_2404_01365_amd as G
import test_layer_abi_cpu as T
calls = {'norm': lambda: T.call_norm(T.mk_norm()), 'norm of many rows': lambda: T.call_norm(T.mk_norm(), rows=5 << 20)}
for dtype in (G.F32, G.BF16):
    C = T.mk_cache(dtype=dtype)
    calls['append %d' % dtype] = lambda C=C: T.append(C, T.mk_batch())
    calls['one chunk %d' % dtype] = lambda C=C: T.attend(C, T.mk_batch(n_prefix=0, max_len=1))
    calls['a token each %d' % dtype] = lambda C=C: T.attend(C, T.mk_batch(n_prefix=2000))
    calls['prompt %d' % dtype] = lambda C=C: T.attend(C, T.mk_batch(cu=(0, 500, 1500), n_prefix=2000, max_len=2000, ld_pages=125))
    calls['short prompt in chunks %d' % dtype] = lambda C=C: T.attend(C, T.mk_batch(cu=(0, 100, 200), n_prefix=2000, max_len=200, ld_pages=13))
for name, call in calls.items():
    shim.shim_fail_at(-1)
    assert call() == G.OK, name
    launches = shim.shim_launches()
    assert launches >= (3 if 'many' in name else 2 if 'each' in name or 'chunks' in name else 1), (name, launches)
    for i in range(launches):
        shim.shim_fail_at(i)
        assert call() == G.EHIP, (name, i)
    print(name, launches)
"""


def test_every_failed_launch_is_reported(tmp_path):
    src, so = str(tmp_path / "shim.c"), str(tmp_path / "shim.so")
    open(src, "w").write(SHIM)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", src, "-o", so])
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, [so, os.environ.get("LD_PRELOAD")])), PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", CALLS, so, os.path.join(ROOT, "tests")], env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
