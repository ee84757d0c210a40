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


# Of the four descriptors around the block, the functions that make them from tensors note beside the fields which card these lie on (None: filled in by hand,
# any), how many tokens a step has and how many pages a table holds.
class griffin_norm(ctypes.Structure):
    _device = None
    _fields_ = [
        ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("kind", ctypes.c_int32), ("eps", ctypes.c_float),
        ("w_offset", ctypes.c_float), ("h_scale", ctypes.c_float), ("y_scale", ctypes.c_float),
        ("w_pre", ctypes.c_void_p), ("b_pre", ctypes.c_void_p), ("w_post", ctypes.c_void_p), ("b_post", ctypes.c_void_p),
    ]


class griffin_kv_cache(ctypes.Structure):
    _device = None
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
        ("dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int64),
        ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
    ]


class griffin_kv_cache_q4(ctypes.Structure):
    _device = None
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
        ("dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("group", ctypes.c_int32), ("n_pages", ctypes.c_int64),
    ]


class griffin_kv_batch(ctypes.Structure):
    _device = _total = _pages = _prefix_pages = None
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
_QP = ctypes.POINTER(griffin_kv_cache_q4)
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
    "griffin_kv_q4_page_bytes": (_sz, [_i32, _i32, _i32, _i32]),
    "griffin_kv_append_q4": (ctypes.c_int, [_QP, _BP] + 4 * [_vp, _i64, _i64] + [_i32, _vp, _vp, _i64, _i32, _i32, _vp]),
    "griffin_kv_read_q4": (ctypes.c_int, [_QP, _BP] + 2 * [_vp, _i64, _i64] + [_vp]),
    "griffin_attention_q4_workspace_bytes": (_sz, [_QP, _BP, _i32]),
    "griffin_attention_q4": (ctypes.c_int, [_QP, _BP, _vp, _i64, _i64, _vp, _i64, _i64, _i32, _f32, _vp, _sz, _vp]),
    "griffin_verify_workspace_bytes": (_sz, [_i32, _i32]),
    "griffin_verify_drafts": (ctypes.c_int, [_vp, _i64, _vp, _i64, _vp, _IP, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
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


_raw_stream = _device = None


def _current_stream() -> int:
    """Handle of PyTorch's current stream.  torch.cuda.current_stream() makes an object for it, which takes as long as a small launch
    (2.7 us); once the runtime is up the handle alone is asked for, where this PyTorch has a call for it."""
    global _raw_stream, _device
    if _raw_stream is None:
        import torch
        if not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        _device = getattr(torch._C, "_cuda_getDevice", None)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if _device is None or _raw_stream is None:
            _device, _raw_stream = (lambda: None), (lambda device: torch.cuda.current_stream().cuda_stream)
    return _raw_stream(_device())


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream() or None
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
# These calls are a few microseconds of work for one token, so their arguments are looked at once: every tensor's shape, type, strides
# and card in one helper.  Descriptors of tensors on the host can be made, and are refused by the calls.
class _Types(dict):
    """PyTorch's type for a griffin_dtype and the other way round; filled when first asked, as the library works without PyTorch."""

    def __missing__(self, key):
        import torch
        if not self:
            self.update({F32: torch.float32, BF16: torch.bfloat16, torch.float32: F32, torch.bfloat16: BF16})
        if key not in self:
            raise TypeError("%s is neither float32 nor bfloat16" % key)
        return self[key]


_TYPE = _Types()


_i32_type = None


def _int32():
    global _i32_type
    if _i32_type is None:
        import torch
        _i32_type = torch.int32
    return _i32_type


def _refuse(what: str, t, shape, dtype, device=None) -> None:
    if dtype is not None and t.dtype is not dtype:
        raise TypeError("%s is %s, not %s" % (what, t.dtype, dtype))
    if t.shape == shape and device is not None and t.get_device() != device:
        raise ValueError("%s is on %s, other tensors of the call on %s" % (what, _place(t.get_device()), _place(device)))
    raise ValueError("%s has shape %s and strides %s; shape %s with a dense last axis is needed"
                     % (what, tuple(t.shape), t.stride(), tuple(shape)))


def _place(device: int) -> str:
    return "the host" if device < 0 else "cuda:%d" % device


def _dense(width: int) -> int:
    return -(-width // 8) * 8


def _row(what: str, t, width: int, dtype, device: int):
    """Address of a vector, or None."""
    if t is None:
        return None
    if t.shape != (width,) or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _refuse(what, t, (width,), dtype, device)
    return t.data_ptr()


def _mat(what: str, t, shape, dtype, device: int):
    """Address and row stride of a matrix, or of None.  A single row has whatever stride it was made with: a dense one is taken."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _refuse(what, t, shape, dtype, device)
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        _refuse(what, t, shape, dtype)
    return t.data_ptr(), ld if shape[0] > 1 else _dense(shape[1])


def _heads(what: str, t, shape, dtype, device: int):
    """Address, token stride and head stride of [tokens][heads][features], or of None."""
    if t is None:
        return None, 0, 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _refuse(what, t, shape, dtype, device)
    ld, hs, one = t.stride()
    if one != 1 and shape[2] > 1:
        _refuse(what, t, shape, dtype)
    return t.data_ptr(), ld if shape[0] > 1 else _dense(shape[2]), hs if shape[1] > 1 else _dense(shape[2])


def norm(w_pre=None, *, b_pre=None, w_post=None, b_post=None, eps: float, w_offset: float = 0.0, kind: int = NORM_RMS,
         h_scale: float = 1.0, y_scale: float = 1.0, d: Optional[int] = None, dtype: Optional[int] = None) -> griffin_norm:
    """Describe the norms around a block ([d] weights and biases; w_pre in front of the next block, w_post behind this one)."""
    some = w_pre if w_pre is not None else w_post
    N = griffin_norm()
    N.d = some.shape[0] if d is None else d
    N.dtype = _TYPE[some.dtype] if dtype is None else dtype
    N._device = None if some is None else some.get_device()
    N.kind, N.eps, N.w_offset, N.h_scale, N.y_scale = kind, eps, w_offset, h_scale, y_scale
    for name, t in (("w_pre", w_pre), ("b_pre", b_pre), ("w_post", w_post), ("b_post", b_post)):
        setattr(N, name, _row("norm: " + name, t, N.d, _TYPE[N.dtype], N._device))
    N._keep = (w_pre, b_pre, w_post, b_post)
    return N


def griffin_norm_residual(N: griffin_norm, h, y=None, h_out=None, x=None, *, gate=None, stream=None) -> None:
    """h_out = h_scale h + y_scale gate N_post(y), x = N_pre(h_out); [rows][d] tensors, gate [d] or [rows][d]."""
    shape, htype, dtype, device = (h.shape[0], N.d), h.dtype, _TYPE[N.dtype], h.get_device() if N._device is None else N._device
    if gate is None:
        at_g, ldg = None, 0
    elif gate.dim() == 2:
        at_g, ldg = _mat("griffin_norm_residual: gate", gate, shape, dtype, device)
    else:
        at_g, ldg = _row("griffin_norm_residual: gate", gate, N.d, dtype, device), 0
    at_h, ldh = _mat("griffin_norm_residual: h", h, shape, htype, device)
    at_y, ldy = _mat("griffin_norm_residual: y", y, shape, dtype, device)
    at_o, ldo = _mat("griffin_norm_residual: h_out", h_out, shape, htype, device)
    at_x, ldx = _mat("griffin_norm_residual: x", x, shape, dtype, device)
    if device < 0:
        raise ValueError("griffin_norm_residual: the tensors lie on the host")
    _check(lib.griffin_norm_residual(N, shape[0], at_h, ldh, _TYPE[htype], at_y, ldy, at_g, ldg, at_o, ldo, at_x, ldx, _stream(stream)),
           "griffin_norm_residual")


def kv_cache(K, V) -> griffin_kv_cache:
    """Describe pools of pages, K and V indexed [page][kv head][token][feature] with the same strides (a pool that holds
    [page][token][kv head][feature] is given as pool.transpose(1, 2))."""
    C = griffin_kv_cache()
    C.dtype = _TYPE[K.dtype]
    C._device, dtype = K.get_device(), _TYPE[C.dtype]
    if K.dim() != 4 or (K.stride(3) != 1 and K.shape[3] > 1):
        _refuse("kv_cache: K", K, (0, 0, 0, 0), None)
    if V.shape != K.shape or V.dtype is not dtype or V.stride() != K.stride() or V.get_device() != C._device:
        _refuse("kv_cache: V", V, K.shape, dtype, C._device)
    C.K, C.V = _ptr(K), _ptr(V)
    C.n_pages, C.kv_heads, C.page_size, C.dim = K.shape
    C.page_stride, C.head_stride, C.token_stride = (st if n > 1 else _dense(C.dim) for n, st in zip(K.shape, K.stride()[:3]))
    C._keep = (K, V)
    return C


def kv_batch(cu_seqlens: Sequence[int], lens, pages, max_len: int, *, prefix_pages=None, n_prefix: int = 0) -> griffin_kv_batch:
    """Describe one step of a batch: its new tokens (host cu_seqlens), and on the device (int32) the sequences' own tokens in the cache,
    their pages [n_seqs][..] and those of the prefix that they share."""
    import torch
    B = griffin_kv_batch()
    B.n_seqs = n = len(cu_seqlens) - 1
    arr = _cu_array(cu_seqlens)
    B.cu_seqlens = ctypes.cast(arr, _IP)
    B._device = device = lens.get_device()
    B.lens = _row("kv_batch: lens", lens, n, torch.int32, device)
    B.pages, B.ld_pages = _mat("kv_batch: pages", pages, (n, pages.shape[-1]), torch.int32, device)
    if n == 1:
        B.ld_pages = pages.shape[1]
    if pages.shape[1] > B.ld_pages:
        raise ValueError("kv_batch: rows of pages overlap")
    B.max_len, B.n_prefix = max_len, n_prefix
    if n_prefix > 0 and prefix_pages is not None:
        B.prefix_pages = _row("kv_batch: prefix_pages", prefix_pages, prefix_pages.numel(), torch.int32, device)
    # what a call compares with max_len and n_prefix, by the cache's page size
    B._total, B._pages, B._prefix_pages = arr[n], pages.shape[1], 0 if prefix_pages is None else prefix_pages.numel()
    B._keep = (arr, lens, pages, prefix_pages)
    return B


def _check_room(where: str, C: griffin_kv_cache, B: griffin_kv_batch, device: int) -> None:
    """`device`: the card of the call's tensors."""
    table = B._device
    if table is not None:
        size = C.page_size
        if B._pages * size < B.max_len or B._prefix_pages * size < B.n_prefix:
            raise ValueError("%s: fewer pages than max_len or n_prefix need" % where)
    if device < 0 or (table != device and table is not None):
        raise ValueError("%s: cache and tensors lie on %s, lens and pages on %s" % (where, _place(device), _place(device if table is None else table)))


# what the arguments of an append, and of an attention, are called in refusals
def _names(where: str, *arguments):
    return (where,) + tuple("%s: %s" % (where, a) for a in arguments)


_APPEND, _APPEND_Q4 = (_names(w, "k", "v", "q", "q_out", "cos", "sin") for w in ("griffin_kv_append", "griffin_kv_append_q4"))
_ATTENTION, _ATTENTION_Q4 = (_names(w, "q", "out", "workspace") for w in ("griffin_attention", "griffin_attention_q4"))
_VERIFY = _names("griffin_verify_drafts", "p", "draft_p", "drafted", "accept_u", "draw_u", "tokens_out", "accepted", "lens", "lens_out", "workspace")


def _append(names, call, C, B: griffin_kv_batch, k, v, q, q_out, cos, sin, style: int, stream) -> None:
    dtype, tokens, dim, device = _TYPE[C.dtype], B._total, C.dim, C._device
    if tokens is None:
        tokens = B.cu_seqlens[B.n_seqs]
    if device is None:
        device = k.get_device()
    kv, heads = (tokens, C.kv_heads, dim), 0 if q is None else q.shape[1]
    at_k, ldk, hsk = _heads(names[1], k, kv, dtype, device)
    at_v, ldv, hsv = _heads(names[2], v, kv, dtype, device)
    at_q, ldq, hsq = _heads(names[3], q, (tokens, heads, dim), dtype, device)
    at_o, ldo, hso = _heads(names[4], q_out, (tokens, heads, dim), dtype, device)
    n_pos = half = 0
    at_c = at_s = None
    if cos is not None:
        n_pos, half = shape = cos.shape
        f32 = _TYPE[F32]
        at_c, ldc = _mat(names[5], cos, shape, f32, device)
        at_s, lds = _mat(names[6], sin, shape, f32, device)
        if n_pos > 1 and (ldc != half or lds != half):
            raise ValueError("%s: rows of cos and sin are not dense" % names[0])
    _check_room(names[0], C, B, device)
    _check(call(C, B, at_k, ldk, hsk, at_v, ldv, hsv, at_q, ldq, hsq, at_o, ldo, hso, heads, at_c, at_s, n_pos, 2 * half, style, _stream(stream)), names[0])


def griffin_kv_append(C: griffin_kv_cache, B: griffin_kv_batch, k, v, *, q=None, q_out=None, cos=None, sin=None,
                      style: int = ROT_HALF, stream=None) -> None:
    """New keys (rotated) and values [tokens][kv_heads][dim] into their pages; queries [tokens][n_heads][dim] rotated into q_out.
    cos, sin: fp32 [positions][rot / 2], None: nothing is rotated."""
    _append(_APPEND, lib.griffin_kv_append, C, B, k, v, q, q_out, cos, sin, style, stream)


def griffin_attention_workspace_bytes(C: griffin_kv_cache, B: griffin_kv_batch, n_heads: int) -> int:
    return int(lib.griffin_attention_workspace_bytes(ctypes.byref(C), ctypes.byref(B), n_heads))


def _attention(names, call, C, B: griffin_kv_batch, q, out, scale, workspace, stream) -> None:
    tokens, dtype, device = B._total, _TYPE[C.dtype], C._device
    if tokens is None:
        tokens = B.cu_seqlens[B.n_seqs]
    if device is None:
        device = q.get_device()
    shape = (tokens, q.shape[1], C.dim)
    at_q, ldq, hsq = _heads(names[1], q, shape, dtype, device)
    at_o, ldo, hso = _heads(names[2], out, shape, dtype, device)
    if workspace is not None and (workspace.get_device() != device or not workspace.is_contiguous()):
        _refuse(names[3], workspace, workspace.shape, None, device)
    _check_room(names[0], C, B, device)
    _check(call(C, B, at_q, ldq, hsq, at_o, ldo, hso, shape[1], shape[2] ** -0.5 if scale is None else scale, _ptr(workspace), _nbytes(workspace),
                _stream(stream)), names[0])


def griffin_attention(C: griffin_kv_cache, B: griffin_kv_batch, q, out, *, scale: Optional[float] = None, workspace=None, stream=None) -> None:
    """out = softmax(scale q K^T) V over the shared prefix and the sequences' own tokens; q, out [tokens][n_heads][dim]."""
    _attention(_ATTENTION, lib.griffin_attention, C, B, q, out, scale, workspace, stream)


# ------------------------------------------------------------------ a cache in 4 bits
def griffin_kv_q4_page_bytes(kv_heads: int, dim: int, page_size: int, group: int = 32) -> int:
    return int(lib.griffin_kv_q4_page_bytes(kv_heads, dim, page_size, group))


def kv_cache_q4(K, V, *, kv_heads: int, dim: int, page_size: int, group: int = 32, dtype) -> griffin_kv_cache_q4:
    """Describe pools of pages in 4 bits, K and V uint8 [page][griffin_kv_q4_page_bytes(..)]; dtype: PyTorch's type of keys, values, queries and
    outputs outside the cache."""
    import torch
    C = griffin_kv_cache_q4()
    C.dtype, C.kv_heads, C.dim, C.page_size, C.group = _TYPE[dtype], kv_heads, dim, page_size, group
    size = griffin_kv_q4_page_bytes(kv_heads, dim, page_size, group)
    if size == 0:
        raise ValueError("kv_cache_q4: no pages of %d heads of %d features, %d tokens, groups of %d" % (kv_heads, dim, page_size, group))
    C._device, shape = K.get_device(), (K.shape[0], size)
    for what, t in (("K", K), ("V", V)):
        if t.shape != shape or t.dtype is not torch.uint8 or t.get_device() != C._device or not t.is_contiguous():
            _refuse("kv_cache_q4: " + what, t, shape, torch.uint8, C._device)
    C.K, C.V, C.n_pages = K.data_ptr(), V.data_ptr(), shape[0]
    C._keep = (K, V)
    return C


def griffin_kv_append_q4(C: griffin_kv_cache_q4, B: griffin_kv_batch, k, v, *, q=None, q_out=None, cos=None, sin=None,
                         style: int = ROT_HALF, stream=None) -> None:
    """griffin_kv_append into a cache in 4 bits."""
    _append(_APPEND_Q4, lib.griffin_kv_append_q4, C, B, k, v, q, q_out, cos, sin, style, stream)


def griffin_kv_read_q4(C: griffin_kv_cache_q4, B: griffin_kv_batch, k=None, v=None, *, stream=None) -> None:
    """What the tokens that griffin_kv_append_q4 writes with this batch stand for, into k and v [tokens][kv_heads][dim] (or one of them)."""
    tokens, device = B._total, C._device
    if tokens is None:
        tokens = B.cu_seqlens[B.n_seqs]
    if device is None:
        device = (v if k is None else k).get_device()
    shape, dtype = (tokens, C.kv_heads, C.dim), _TYPE[C.dtype]
    at_k, ldk, hsk = _heads("griffin_kv_read_q4: k", k, shape, dtype, device)
    at_v, ldv, hsv = _heads("griffin_kv_read_q4: v", v, shape, dtype, device)
    _check_room("griffin_kv_read_q4", C, B, device)
    _check(lib.griffin_kv_read_q4(C, B, at_k, ldk, hsk, at_v, ldv, hsv, _stream(stream)), "griffin_kv_read_q4")


def griffin_attention_q4_workspace_bytes(C: griffin_kv_cache_q4, B: griffin_kv_batch, n_heads: int) -> int:
    return int(lib.griffin_attention_q4_workspace_bytes(ctypes.byref(C), ctypes.byref(B), n_heads))


def griffin_attention_q4(C: griffin_kv_cache_q4, B: griffin_kv_batch, q, out, *, scale: Optional[float] = None, workspace=None, stream=None) -> None:
    """griffin_attention over a cache in 4 bits."""
    _attention(_ATTENTION_Q4, lib.griffin_attention_q4, C, B, q, out, scale, workspace, stream)


# ------------------------------------------------------------------ drafted tokens
def cu_seqlens(values: Sequence[int]):
    """A batch's host array of sequence ends, made once where a call is made many times."""
    return _cu_array(values)


def griffin_verify_workspace_bytes(n_seqs: int, vocab: int) -> int:
    return int(lib.griffin_verify_workspace_bytes(n_seqs, vocab))


def griffin_verify_drafts(cu_seqlens, p, drafted, accept_u, draw_u, tokens_out, accepted, *, draft_p=None, lens=None, lens_out=None, workspace=None,
                          stream=None) -> None:
    """Keeps the drafted tokens that the target's probabilities p [rows][vocab] allow and draws the one behind them.  cu_seqlens: a sequence of ints or
    what cu_seqlens() made of one; drafted, accept_u, tokens_out [rows]; draw_u, accepted, lens, lens_out [sequences].  tokens_out shares no element with
    drafted."""
    cu = cu_seqlens if isinstance(cu_seqlens, ctypes.Array) else _cu_array(cu_seqlens)
    n, device, f32, i32, names = len(cu) - 1, p.get_device(), _TYPE[F32], _int32(), _VERIFY
    if n < 1:
        raise ValueError("griffin_verify_drafts: no sequences")
    rows = cu[n]
    shape = (rows, p.shape[-1])
    at_p, ldp = _mat(names[1], p, shape, f32, device)
    at_q, ldq = _mat(names[2], draft_p, shape, f32, device)
    if rows == 1:
        ldp = ldq = shape[1]
    at_d, at_u = _row(names[3], drafted, rows, i32, device), _row(names[4], accept_u, rows, f32, device)
    at_r, at_t = _row(names[5], draw_u, n, f32, device), _row(names[6], tokens_out, rows, i32, device)
    at_a, at_l, at_o = _row(names[7], accepted, n, i32, device), _row(names[8], lens, n, i32, device), _row(names[9], lens_out, n, i32, device)
    if workspace is not None and (workspace.get_device() != device or not workspace.is_contiguous()):
        _refuse(names[10], workspace, workspace.shape, None, device)
    if device < 0:
        raise ValueError("griffin_verify_drafts: the tensors lie on the host")
    _check(lib.griffin_verify_drafts(at_p, ldp, at_q, ldq, at_d, cu, n, shape[1], at_u, at_r, at_t, at_a, at_l, at_o, _ptr(workspace), _nbytes(workspace),
                                     _stream(stream)), names[0])
