"""Thin Python binding of libgriffin.so (the C ABI declared in include/griffin.h).

Argument marshalling only: every step of the path runs in the library's HIP kernels.
PyTorch supplies device memory (``tensor.data_ptr()``) and the current stream; nothing here
computes, and there is no CPU or PyTorch fallback -- if the library is missing the import
fails.  Function names match the C entry points.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgriffin.so")

OK, EINVAL, ESHAPE, EWORKSPACE, EUNSUPPORTED, EHIP = range(6)
ACT_SILU, ACT_GELU_TANH, ACT_RELU = 0, 1, 2
F32, BF16 = 0, 1
MAX_SEQS, MAX_BATCH = 256, 64
NORM_RMS, NORM_LAYER = 0, 1
ROT_HALF, ROT_PAIRS = 0, 1


class GriffinError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib.griffin_status_string(status).decode()
        if status == EHIP:
            msg += " (" + lib.griffin_last_hip_error().decode() + ")"
        super().__init__("%s: %s [status %d]" % (where, msg, status))


class griffin_layer(ctypes.Structure):
    _fields_ = [
        ("d", ctypes.c_int32), ("n", ctypes.c_int32), ("dtype", ctypes.c_int32), ("act", ctypes.c_int32),
        ("Wg", ctypes.c_void_p), ("W1", ctypes.c_void_p), ("W2", ctypes.c_void_p),
        ("ld", ctypes.c_int64),
        ("bg", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("b2", ctypes.c_void_p),
        ("W2t", ctypes.c_void_p), ("ldt", ctypes.c_int64),
    ]


class griffin_norm(ctypes.Structure):
    _fields_ = [
        ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("kind", ctypes.c_int32), ("eps", ctypes.c_float),
        ("w_offset", ctypes.c_float), ("h_scale", ctypes.c_float), ("y_scale", ctypes.c_float),
        ("w_pre", ctypes.c_void_p), ("b_pre", ctypes.c_void_p), ("w_post", ctypes.c_void_p), ("b_post", ctypes.c_void_p),
    ]


class griffin_kv_cache(ctypes.Structure):
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
        ("dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int64),
        ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
    ]


class griffin_kv_batch(ctypes.Structure):
    _fields_ = [
        ("cu_seqlens", ctypes.POINTER(ctypes.c_int32)), ("n_seqs", ctypes.c_int32), ("max_len", ctypes.c_int32),
        ("lens", ctypes.c_void_p), ("pages", ctypes.c_void_p), ("ld_pages", ctypes.c_int64),
        ("n_prefix", ctypes.c_int32), ("prefix_pages", ctypes.c_void_p),
    ]


def _load() -> ctypes.CDLL:
    # libgriffin.so needs libamdhip64.so.7.  PyTorch ships its own copy of that runtime; a
    # process must not end up with two HIP runtimes (the second one sees no device), so
    # PyTorch's is loaded first and the dynamic loader hands the same object to libgriffin.
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "%s is missing: build it with `python paper_2404_01365_amd/build.py` "
            "(there is no fallback path)" % LIB_PATH)
    return ctypes.CDLL(LIB_PATH)


lib = _load()

_vp, _i32, _i64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_LP = ctypes.POINTER(griffin_layer)
_IP = ctypes.POINTER(ctypes.c_int32)
_NP, _CP, _BP = (ctypes.POINTER(t) for t in (griffin_norm, griffin_kv_cache, griffin_kv_batch))
_f32 = ctypes.c_float

_SIGS = {
    "griffin_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "griffin_last_hip_error": (ctypes.c_char_p, []),
    "griffin_version": (ctypes.c_char_p, []),
    "griffin_k_from_fraction": (_i32, [_i32, ctypes.c_double]),
    "griffin_prefill_workspace_bytes": (_sz, [_LP, _i64, _i32, _i32]),
    "griffin_prefill_select": (ctypes.c_int, [_LP, _vp, _i64, _IP, _i32, _i32, _vp, _vp, _vp, _i64, _vp, _sz, _vp]),
    "griffin_topk": (ctypes.c_int, [_vp, _i32, _i32, _i32, _vp, _vp]),
    "griffin_stat_shared": (ctypes.c_int, [_vp, _IP, _i32, _i32, _vp, _vp]),
    "griffin_compact": (ctypes.c_int, [_LP, _vp, _i32, _LP, _vp]),
    "griffin_weight_norm_score": (ctypes.c_int, [_LP, _vp, _vp]),
    "griffin_select_sampled_workspace_bytes": (_sz, [_i32, _i32]),
    "griffin_select_sampled": (ctypes.c_int, [_vp, _vp, _i32, _i32, _i32, _vp, _vp, _sz, _vp]),
    "griffin_jaccard": (ctypes.c_int, [_vp, _i32, _i32, _vp, _vp]),
    "griffin_decode_workspace_bytes": (_sz, [_i32, _i32, _i32]),
    "griffin_trace_next_decode": (ctypes.c_int, [_vp, _vp, _vp]),
    "griffin_prompt_out_workspace_bytes": (_sz, [_i64, _i32, _i32]),
    "griffin_ff_prompt_out": (ctypes.c_int, [_vp, _i64, _i64, _i32, _i32, _i32, _vp, _i64, _vp, _vp, _i64, _vp, _sz, _vp]),
    "griffin_prompt_phase_workspace_bytes": (_sz, [_LP, _i64, _i32]),
    "griffin_prompt_phase": (ctypes.c_int, [_LP, _vp, _i64, _vp, _i64, _IP, _i32, _i32, _vp, _vp, _vp, _i64, _vp, _sz, _vp]),
    "griffin_ff_decode": (ctypes.c_int, [_LP, _vp, _vp, _i32, _vp, _sz, _vp]),
    "griffin_ff_decode_static_max_bytes": (_sz, []),
    "griffin_ff_decode_static": (ctypes.c_int, [_LP, _vp, _vp, _i32, _vp]),
    "griffin_ff_decode_multi": (ctypes.c_int, [_LP, _i32, _vp, _vp, _vp, _sz, _vp]),
    "griffin_ff_decode_indexed": (ctypes.c_int, [_LP, _vp, _i32, _i32, _vp, _vp, _vp, _sz, _vp]),
    "griffin_index_sets_bytes": (_sz, [_i32, _i32]),
    "griffin_index_sets_build": (ctypes.c_int, [_vp, _i32, _i32, _i32, _vp, _sz, _vp]),
    "griffin_ff_decode_indexed_sets": (ctypes.c_int, [_LP, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "griffin_norm_residual": (ctypes.c_int, [_NP, _i64, _vp, _i64, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp]),
    "griffin_kv_append": (ctypes.c_int, [_CP, _BP] + 4 * [_vp, _i64, _i64] + [_i32, _vp, _vp, _i64, _i32, _i32, _vp]),
    "griffin_attention_workspace_bytes": (_sz, [_CP, _BP, _i32]),
    "griffin_attention": (ctypes.c_int, [_CP, _BP, _vp, _i64, _i64, _vp, _i64, _i64, _i32, _f32, _vp, _sz, _vp]),
}
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

EXPORTS = tuple(_SIGS)


# ------------------------------------------------------------------ marshalling helpers
def _ptr(t) -> Optional[int]:
    """Device (or raw integer) address of a tensor; None stays NULL."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise GriffinError(status, where)


def layer(W1, W2, Wg=None, *, act: int, dtype: Optional[int] = None, bg=None, b1=None, b2=None,
          d: Optional[int] = None, n: Optional[int] = None, ld: Optional[int] = None, W2t=None) -> griffin_layer:
    """Describe one FF block held in torch tensors ([n][d] neuron-major, contiguous rows).
    W2t: optional [d][ldt] copy of W2 in the paper's orientation (W2 may then be None)."""
    import torch
    if dtype is None:
        dtype = BF16 if W1.dtype == torch.bfloat16 else F32
    L = griffin_layer()
    L.n = W1.shape[0] if n is None else n
    L.d = W1.shape[1] if d is None else d
    L.ld = W1.stride(0) if ld is None else ld
    L.dtype, L.act = dtype, act
    L.Wg, L.W1, L.W2 = _ptr(Wg), _ptr(W1), _ptr(W2)
    L.bg, L.b1, L.b2 = _ptr(bg), _ptr(b1), _ptr(b2)
    L.W2t = _ptr(W2t)
    L.ldt = 0 if W2t is None else W2t.stride(0)
    # keep the tensors alive as long as the descriptor
    L._keep = (W1, W2, Wg, bg, b1, b2, W2t)
    return L


def _cu_array(cu_seqlens: Sequence[int]):
    arr = (ctypes.c_int32 * len(cu_seqlens))(*[int(v) for v in cu_seqlens])
    return arr


# ------------------------------------------------------------------ entry points
def griffin_version() -> str:
    return lib.griffin_version().decode()


def griffin_status_string(status: int) -> str:
    return lib.griffin_status_string(status).decode()


def griffin_k_from_fraction(d_ff: int, keep: float) -> int:
    return int(lib.griffin_k_from_fraction(d_ff, keep))


def griffin_prefill_workspace_bytes(L: griffin_layer, total_tokens: int, n_seqs: int = 1,
                                    have_z_out: bool = False) -> int:
    return int(lib.griffin_prefill_workspace_bytes(ctypes.byref(L), total_tokens, n_seqs, int(have_z_out)))


def griffin_prefill_select(L: griffin_layer, X, cu_seqlens: Sequence[int], k: int, idx_out, *,
                           s_out=None, Z_out=None, workspace, ldx: Optional[int] = None,
                           ldz: Optional[int] = None, stream=None) -> None:
    n_seqs = len(cu_seqlens) - 1
    if ldx is None:
        ldx = X.stride(0) if X is not None and X.dim() == 2 else L.d
    if ldz is None:
        ldz = Z_out.stride(0) if Z_out is not None else 0
    st = lib.griffin_prefill_select(ctypes.byref(L), _ptr(X), ldx, _cu_array(cu_seqlens), n_seqs, k,
                                    _ptr(idx_out), _ptr(s_out), _ptr(Z_out), ldz,
                                    _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(st, "griffin_prefill_select")


def griffin_topk(scores, k: int, idx_out, *, stream=None) -> None:
    n_rows, n = (1, scores.shape[0]) if scores.dim() == 1 else scores.shape
    _check(lib.griffin_topk(_ptr(scores), n_rows, n, k, _ptr(idx_out), _stream(stream)), "griffin_topk")


def griffin_stat_shared(s, cu_seqlens: Sequence[int], sbar_out, *, stream=None) -> None:
    n_seqs = len(cu_seqlens) - 1
    _check(lib.griffin_stat_shared(_ptr(s), _cu_array(cu_seqlens), n_seqs, s.shape[-1], _ptr(sbar_out),
                                   _stream(stream)), "griffin_stat_shared")


def griffin_weight_norm_score(L: griffin_layer, score_out, *, stream=None) -> None:
    _check(lib.griffin_weight_norm_score(ctypes.byref(L), _ptr(score_out), _stream(stream)),
           "griffin_weight_norm_score")


def griffin_select_sampled_workspace_bytes(n: int, k_top: int) -> int:
    return int(lib.griffin_select_sampled_workspace_bytes(n, k_top))


def griffin_select_sampled(s, e, k: int, k_top: int, idx_out, *, workspace, stream=None) -> None:
    _check(lib.griffin_select_sampled(_ptr(s), _ptr(e), s.shape[-1], k, k_top, _ptr(idx_out),
                                      _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "griffin_select_sampled")


def griffin_jaccard(idx, out, *, stream=None) -> None:
    n_sets, k = idx.shape
    _check(lib.griffin_jaccard(_ptr(idx), n_sets, k, _ptr(out), _stream(stream)), "griffin_jaccard")


def griffin_compact(L: griffin_layer, idx, k: int, C: griffin_layer, *, stream=None) -> None:
    _check(lib.griffin_compact(ctypes.byref(L), _ptr(idx), k, ctypes.byref(C), _stream(stream)),
           "griffin_compact")


def griffin_decode_workspace_bytes(d: int, n: int, batch: int = 1) -> int:
    return int(lib.griffin_decode_workspace_bytes(d, n, batch))


def griffin_ff_decode(C: griffin_layer, x, y, batch: int = 1, *, workspace, stream=None) -> None:
    _check(lib.griffin_ff_decode(ctypes.byref(C), _ptr(x), _ptr(y), batch, _ptr(workspace),
                                 _nbytes(workspace), _stream(stream)), "griffin_ff_decode")


def griffin_ff_decode_static_max_bytes() -> int:
    return int(lib.griffin_ff_decode_static_max_bytes())


def griffin_ff_decode_static(C: griffin_layer, x, y, batch: int = 1, *, stream=None) -> None:
    """griffin_ff_decode with the partial rows in the library's own device array (no workspace)."""
    _check(lib.griffin_ff_decode_static(ctypes.byref(C), _ptr(x), _ptr(y), batch, _stream(stream)),
           "griffin_ff_decode_static")


def griffin_ff_decode_multi(Cs: Sequence[griffin_layer], x, y, *, workspace, stream=None) -> None:
    arr = (griffin_layer * len(Cs))(*Cs)
    _check(lib.griffin_ff_decode_multi(arr, len(Cs), _ptr(x), _ptr(y), _ptr(workspace),
                                       _nbytes(workspace), _stream(stream)), "griffin_ff_decode_multi")


def griffin_ff_decode_indexed(L: griffin_layer, idx, k: int, batch: int, x, y, *, workspace,
                              stream=None) -> None:
    _check(lib.griffin_ff_decode_indexed(ctypes.byref(L), _ptr(idx), k, batch, _ptr(x), _ptr(y),
                                         _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "griffin_ff_decode_indexed")


def griffin_index_sets_bytes(n: int, batch: int) -> int:
    return int(lib.griffin_index_sets_bytes(n, batch))


def griffin_index_sets_build(idx, k: int, batch: int, n: int, sets, *, stream=None) -> None:
    _check(lib.griffin_index_sets_build(_ptr(idx), k, batch, n, _ptr(sets), _nbytes(sets), _stream(stream)),
           "griffin_index_sets_build")


def griffin_ff_decode_indexed_sets(L: griffin_layer, idx, k: int, sets, batch: int, x, y, *, workspace,
                                   stream=None) -> None:
    _check(lib.griffin_ff_decode_indexed_sets(ctypes.byref(L), _ptr(idx), k, _ptr(sets), batch, _ptr(x), _ptr(y),
                                              _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "griffin_ff_decode_indexed_sets")


def griffin_prompt_phase_workspace_bytes(L: griffin_layer, total_tokens: int, n_seqs: int) -> int:
    return int(lib.griffin_prompt_phase_workspace_bytes(ctypes.byref(L), total_tokens, n_seqs))


def griffin_prompt_phase(L: griffin_layer, W2p, X, cu_seqlens: Sequence[int], k: int, idx_out, Y, *,
                         s_out=None, workspace, ldx: Optional[int] = None, stream=None) -> None:
    """Selection and the prompt's own output from one Z (W2p is the paper's W_2, [d][d_ff])."""
    n_seqs = len(cu_seqlens) - 1
    if ldx is None:
        ldx = X.stride(0) if X is not None and X.dim() == 2 else L.d
    st = lib.griffin_prompt_phase(ctypes.byref(L), _ptr(W2p), W2p.stride(0), _ptr(X), ldx, _cu_array(cu_seqlens),
                                  n_seqs, k, _ptr(idx_out), _ptr(s_out), _ptr(Y), Y.stride(0),
                                  _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(st, "griffin_prompt_phase")


def griffin_trace_next_decode(event_begin: Optional[int], event_mid: Optional[int],
                              event_end: Optional[int]) -> None:
    """Arm one-shot hipEvent_t handles before / between / after the next decode call's two kernels."""
    _check(lib.griffin_trace_next_decode(event_begin, event_mid, event_end), "griffin_trace_next_decode")


def griffin_prompt_out_workspace_bytes(total_tokens: int, d_ff: int, d: int) -> int:
    return int(lib.griffin_prompt_out_workspace_bytes(total_tokens, d_ff, d))


def griffin_ff_prompt_out(Z, W2p, Y, *, b2=None, dtype: Optional[int] = None, workspace=None, stream=None) -> None:
    """Y = Z W2p^T + b2 for the prompt rows (W2p is the paper's W_2, [d][d_ff])."""
    import torch
    if dtype is None:
        dtype = BF16 if W2p.dtype == torch.bfloat16 else F32
    _check(lib.griffin_ff_prompt_out(_ptr(Z), Z.stride(0), Z.shape[0], Z.shape[1], W2p.shape[0], dtype,
                                     _ptr(W2p), W2p.stride(0), _ptr(b2), _ptr(Y), Y.stride(0),
                                     _ptr(workspace), _nbytes(workspace), _stream(stream)), "griffin_ff_prompt_out")


# ------------------------------------------------------------------ around the block
def _dtype_of(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError("%s is neither float32 nor bfloat16" % t.dtype)


def _shape(what: str, t, *sizes) -> None:
    """Sizes (None: any) of a tensor whose last axis is dense; the library sees pointers and strides only."""
    if t.dim() != len(sizes) or any(n is not None and m != n for m, n in zip(t.shape, sizes)) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError("%s: shape %s, strides %s" % (what, tuple(t.shape), t.stride()))


def _strides(t, width: int):
    """A tensor's strides but the last; an axis of one element has whatever stride it was made with, so a dense one is taken."""
    if t is None:
        return (0, 0)
    return tuple(st if n > 1 else -(-width // 8) * 8 for n, st in zip(t.shape[:-1], t.stride()))


def _same_type(what: str, dtype: int, *tensors) -> None:
    for t in tensors:
        if t is not None and _dtype_of(t) != dtype:
            raise TypeError("%s: %s beside %s" % (what, t.dtype, "bfloat16" if dtype == BF16 else "float32"))


def norm(w_pre=None, *, b_pre=None, w_post=None, b_post=None, eps: float, w_offset: float = 0.0, kind: int = NORM_RMS,
         h_scale: float = 1.0, y_scale: float = 1.0, d: Optional[int] = None, dtype: Optional[int] = None) -> griffin_norm:
    """Describe the norms around a block ([d] weights and biases; w_pre in front of the next block, w_post behind this one)."""
    some = w_pre if w_pre is not None else w_post
    N = griffin_norm()
    N.d = some.shape[0] if d is None else d
    N.dtype = _dtype_of(some) if dtype is None else dtype
    for name, t in (("w_pre", w_pre), ("b_pre", b_pre), ("w_post", w_post), ("b_post", b_post)):
        if t is not None:
            _shape("norm: " + name, t, N.d)
            _same_type("norm: " + name, N.dtype, t)
    N.kind, N.eps, N.w_offset, N.h_scale, N.y_scale = kind, eps, w_offset, h_scale, y_scale
    N.w_pre, N.b_pre, N.w_post, N.b_post = _ptr(w_pre), _ptr(b_pre), _ptr(w_post), _ptr(b_post)
    N._keep = (w_pre, b_pre, w_post, b_post)
    return N


def griffin_norm_residual(N: griffin_norm, h, y=None, h_out=None, x=None, *, gate=None, stream=None) -> None:
    """h_out = h_scale h + y_scale gate N_post(y), x = N_pre(h_out); [rows][d] tensors, gate [d] or [rows][d]."""
    rows = h.shape[0]
    for name, t in (("h", h), ("y", y), ("h_out", h_out), ("x", x)):
        if t is not None:
            _shape("griffin_norm_residual: " + name, t, rows, N.d)
    h_dtype = _dtype_of(h)
    _same_type("griffin_norm_residual", N.dtype, y, gate, x)
    _same_type("griffin_norm_residual", h_dtype, h_out)
    ld = lambda t: _strides(t, N.d)[0]  # noqa: E731
    ldg = 0
    if gate is not None:
        _shape("griffin_norm_residual: gate", gate, *((rows, N.d) if gate.dim() == 2 else (N.d,)))
        ldg = ld(gate) if gate.dim() == 2 else 0
    _check(lib.griffin_norm_residual(ctypes.byref(N), rows, _ptr(h), ld(h), h_dtype, _ptr(y), ld(y), _ptr(gate), ldg, _ptr(h_out),
                                     ld(h_out), _ptr(x), ld(x), _stream(stream)), "griffin_norm_residual")


def kv_cache(K, V) -> griffin_kv_cache:
    """Describe pools of pages, K and V indexed [page][kv head][token][feature] with the same strides (a pool that holds
    [page][token][kv head][feature] is given as pool.transpose(1, 2))."""
    _shape("kv_cache: K", K, None, None, None, None)
    _shape("kv_cache: V", V, *K.shape)
    if K.stride() != V.stride():
        raise ValueError("kv_cache: K and V have strides %s and %s" % (K.stride(), V.stride()))
    C = griffin_kv_cache()
    C.K, C.V, C.dtype = _ptr(K), _ptr(V), _dtype_of(K)
    _same_type("kv_cache", C.dtype, V)
    C.n_pages, C.kv_heads, C.page_size, C.dim = K.shape
    C.page_stride, C.head_stride, C.token_stride = _strides(K, C.dim)
    C._keep = (K, V)
    return C


def kv_batch(cu_seqlens: Sequence[int], lens, pages, max_len: int, *, prefix_pages=None, n_prefix: int = 0) -> griffin_kv_batch:
    """Describe one step of a batch: its new tokens (host cu_seqlens), and on the device (int32) the sequences' own tokens in the cache,
    their pages [n_seqs][..] and those of the prefix that they share."""
    import torch
    B = griffin_kv_batch()
    B.n_seqs = len(cu_seqlens) - 1
    for name, t in (("lens", lens), ("pages", pages), ("prefix_pages", prefix_pages)):
        if t is not None and t.dtype != torch.int32:
            raise TypeError("kv_batch: %s is %s, not int32" % (name, t.dtype))
    _shape("kv_batch: lens", lens, B.n_seqs)
    _shape("kv_batch: pages", pages, B.n_seqs, None)
    arr = _cu_array(cu_seqlens)
    B.cu_seqlens = ctypes.cast(arr, _IP)
    B.max_len, B.lens, B.pages = max_len, _ptr(lens), _ptr(pages)
    B.ld_pages = pages.shape[1] if B.n_seqs == 1 else pages.stride(0)
    if pages.shape[1] > B.ld_pages:
        raise ValueError("kv_batch: rows of pages overlap")
    B.n_prefix, B.prefix_pages = n_prefix, _ptr(prefix_pages) if n_prefix > 0 else None
    B._total, B._prefix_room = int(cu_seqlens[-1]), 0 if prefix_pages is None else prefix_pages.numel()
    B._row_pages = pages.shape[1]
    B._keep = (arr, lens, pages, prefix_pages)
    return B


def _check_room(where: str, C: griffin_kv_cache, B: griffin_kv_batch) -> None:
    if B._row_pages * C.page_size < B.max_len or B._prefix_room * C.page_size < B.n_prefix:
        raise ValueError("%s: fewer pages than max_len or n_prefix need" % where)


def griffin_kv_append(C: griffin_kv_cache, B: griffin_kv_batch, k, v, *, q=None, q_out=None, cos=None, sin=None,
                      style: int = ROT_HALF, stream=None) -> None:
    """New keys (rotated) and values [tokens][kv_heads][dim] into their pages; queries [tokens][n_heads][dim] rotated into q_out.
    cos, sin: fp32 [positions][rot / 2], None: nothing is rotated."""
    where = "griffin_kv_append"
    heads = 0 if q is None else q.shape[1]
    for name, t, n in (("k", k, C.kv_heads), ("v", v, C.kv_heads), ("q", q, heads), ("q_out", q_out, heads)):
        if t is not None:
            _shape(where + ": " + name, t, B._total, n, C.dim)
    _same_type(where, C.dtype, k, v, q, q_out)
    _check_room(where, C, B)
    rot = n_pos = 0
    if cos is not None:
        import torch
        n_pos, rot = cos.shape[0], 2 * cos.shape[1]
        if cos.dtype != torch.float32 or sin.dtype != torch.float32 or sin.shape != cos.shape or not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError(where + ": cos and sin are not two dense float32 tables of one shape")
    st = lambda t: _strides(t, C.dim)  # noqa: E731
    _check(lib.griffin_kv_append(ctypes.byref(C), ctypes.byref(B), _ptr(k), *st(k), _ptr(v), *st(v), _ptr(q), *st(q), _ptr(q_out), *st(q_out),
                                 heads, _ptr(cos), _ptr(sin), n_pos, rot, style, _stream(stream)), where)


def griffin_attention_workspace_bytes(C: griffin_kv_cache, B: griffin_kv_batch, n_heads: int) -> int:
    return int(lib.griffin_attention_workspace_bytes(ctypes.byref(C), ctypes.byref(B), n_heads))


def griffin_attention(C: griffin_kv_cache, B: griffin_kv_batch, q, out, *, scale: Optional[float] = None, workspace=None, stream=None) -> None:
    """out = softmax(scale q K^T) V over the shared prefix and the sequences' own tokens; q, out [tokens][n_heads][dim]."""
    where = "griffin_attention"
    heads = q.shape[1]
    _shape(where + ": q", q, B._total, heads, C.dim)
    _shape(where + ": out", out, B._total, heads, C.dim)
    _same_type(where, C.dtype, q, out)
    _check_room(where, C, B)
    (ldq, hsq), (ldo, hso) = _strides(q, C.dim), _strides(out, C.dim)
    _check(lib.griffin_attention(ctypes.byref(C), ctypes.byref(B), _ptr(q), ldq, hsq, _ptr(out), ldo, hso, heads,
                                 C.dim ** -0.5 if scale is None else scale, _ptr(workspace), _nbytes(workspace), _stream(stream)), where)
