"""Thin ctypes binding of the C ABI in include/dart.h.

Argument marshalling only: every step runs in the HIP kernels of
libdart_hip.so.  PyTorch supplies device memory and the current stream.  If the
library is missing this module raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch


LIB = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdart_hip.so")

DART_OK = 0
DART_ERR_NULL, DART_ERR_SHAPE, DART_ERR_BUDGET, DART_ERR_DTYPE = -1, -2, -3, -4
DART_ERR_WORKSPACE, DART_ERR_ALIGN, DART_ERR_HIP, DART_ERR_DEVICE = -5, -6, -7, -8
DART_ERR_STATIC_LIMIT = -9
DART_F32, DART_BF16 = 0, 1
DART_PIVOT_MAX_L1, DART_PIVOT_MIN_L1, DART_PIVOT_GIVEN, DART_PIVOT_RANDOM = 0, 1, 2, 3
DART_SCORE_PER_PIVOT, DART_SCORE_MIN, DART_SCORE_MAX = 0, 1, 2

EXPORTS = ("dart_workspace_bytes", "dart_select_pivots", "dart_duplication_scores",
           "dart_topk_keep", "dart_gather_compact", "dart_compact_sequences", "dart_reduce",
           "dart_reduce_profiled", "dart_reduce_static", "dart_static_scratch_bytes",
           "dart_device_status_static", "dart_probe_mfma_dot32", "dart_score_tile_shape",
           "dart_score_tile_shape_first_read", "dart_reduce_with_norms",
           "dart_device_status", "dart_score_tolerance", "dart_norm_rotate",
           "dart_norm_rotate_append", "dart_attend_workspace_bytes", "dart_attend",
           "dart_append_4bit", "dart_read_4bit", "dart_attend_4bit_workspace_bytes", "dart_attend_4bit",
           "dart_attend_weights_workspace_bytes", "dart_attend_weights", "dart_evict_most",
           "dart_evict_workspace_bytes", "dart_evict",
           "dart_strerror")


class DartDesc(C.Structure):
    """Mirror of `struct dart_desc`."""
    _fields_ = [("B", C.c_int32), ("D", C.c_int32), ("P", C.c_int32), ("N", C.c_int32),
                ("cu_seqlens", C.c_void_p), ("total_N", C.c_int32), ("max_N", C.c_int32),
                ("ld", C.c_int64), ("dtype", C.c_int32), ("K", C.c_int32),
                ("keep_num", C.c_int32), ("keep_den", C.c_int32), ("pivot_mode", C.c_int32),
                ("score_mode", C.c_int32), ("P_ext", C.c_int32), ("ext_ld", C.c_int64),
                ("ext_pivots", C.c_void_p), ("span_start", C.c_void_p), ("X_rows", C.c_int32),
                ("seed", C.c_uint64)]


class DartRowTensor(C.Structure):
    """Mirror of `struct dart_row_tensor`."""
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("row_bytes", C.c_int64),
                ("src_ld_bytes", C.c_int64), ("dst_ld_bytes", C.c_int64)]


class DartRotation(C.Structure):
    """Mirror of `struct dart_rotation`."""
    _fields_ = [("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32),
                ("rot", C.c_int32), ("interleaved", C.c_int32), ("planes", C.c_int32),
                ("sections", C.c_int32 * 4), ("inv_freq", C.c_void_p), ("q_weight", C.c_void_p),
                ("k_weight", C.c_void_p), ("eps", C.c_float), ("scale", C.c_float)]


class DartCache(C.Structure):
    """Mirror of `struct dart_cache`."""
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                ("dtype", C.c_int32), ("T", C.c_int32), ("max_q", C.c_int32),
                ("max_kv", C.c_int32), ("cu_q", C.c_void_p), ("kv_len", C.c_void_p),
                ("pages", C.c_void_p), ("pages_ld", C.c_int32), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("page_ld", C.c_int64), ("head_ld", C.c_int64),
                ("row_ld", C.c_int64), ("groups", C.c_int32), ("max_prefix", C.c_int32),
                ("group_cu", C.c_void_p), ("prefix_pages", C.c_void_p),
                ("prefix_len", C.c_void_p), ("prefix_ld", C.c_int32), ("pages_n", C.c_int32),
                ("prefix_n", C.c_int32)]


class DartEviction(C.Structure):
    """Mirror of `struct dart_eviction`."""
    _fields_ = [("budget", C.c_int32), ("ratio_num", C.c_int32), ("ratio_den", C.c_int32),
                ("first", C.c_int32), ("recent", C.c_int32)]


class DartError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


_lib = None


def lib():
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB):
            raise RuntimeError(f"{LIB} is missing: run `python -m paper_2502_11494_amd.build`")
        L = C.CDLL(LIB)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        dp = C.POINTER(DartDesc)
        L.dart_workspace_bytes.argtypes = [dp]
        L.dart_workspace_bytes.restype = sz
        L.dart_select_pivots.argtypes = [dp, vp, vp, i32, i64, vp, vp, vp, sz, vp]
        L.dart_duplication_scores.argtypes = [dp, vp, vp, vp, vp, sz, vp]
        L.dart_topk_keep.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dart_gather_compact.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dart_compact_sequences.argtypes = [dp, vp, vp, i32, C.POINTER(DartRowTensor), vp, i32,
                                             i64, vp, i64, vp, vp, vp, sz, vp]
        L.dart_reduce.argtypes = [dp, vp, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dart_reduce_profiled.argtypes = L.dart_reduce.argtypes + [C.POINTER(vp)]
        L.dart_reduce_with_norms.argtypes = [dp, vp, vp, i32, i64, vp, C.c_double, vp, vp, vp, vp,
                                             vp, vp, vp, vp, sz, vp]
        L.dart_device_status.argtypes = [dp, vp, vp]
        L.dart_reduce_static.argtypes = [dp, vp, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp]
        L.dart_score_tile_shape.argtypes = [dp, C.POINTER(i32), C.POINTER(i32)]
        L.dart_score_tile_shape_first_read.argtypes = [dp, C.POINTER(i32), C.POINTER(i32)]
        L.dart_static_scratch_bytes.argtypes = []
        L.dart_static_scratch_bytes.restype = sz
        L.dart_device_status_static.argtypes = [dp, vp]
        L.dart_probe_mfma_dot32.argtypes = [vp, vp, vp, i32, vp]
        rp, cp, f32 = C.POINTER(DartRotation), C.POINTER(DartCache), C.c_float
        L.dart_norm_rotate.argtypes = [rp, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp]
        L.dart_norm_rotate_append.argtypes = [rp, cp, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64,
                                              vp, i64, vp, vp, vp, vp, vp]
        L.dart_attend_workspace_bytes.argtypes = [cp]
        L.dart_attend_workspace_bytes.restype = sz
        L.dart_attend.argtypes = [cp, vp, i64, vp, vp, f32, i32, vp, i64, vp, vp, sz, vp, vp]
        L.dart_append_4bit.argtypes = [cp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp]
        L.dart_read_4bit.argtypes = [cp, vp, vp, vp, vp, vp, i64, vp, i64, vp, vp]
        L.dart_attend_4bit_workspace_bytes.argtypes = [cp]
        L.dart_attend_4bit_workspace_bytes.restype = sz
        L.dart_attend_4bit.argtypes = [cp, vp, i64, vp, vp, vp, vp, f32, i32, vp, i64, vp, vp, sz, vp, vp]
        ep = C.POINTER(DartEviction)
        L.dart_attend_weights_workspace_bytes.argtypes = [cp, i32]
        L.dart_attend_weights_workspace_bytes.restype = sz
        L.dart_attend_weights.argtypes = [cp, vp, i64, vp, vp, vp, f32, i32, f32, vp, vp, sz, vp, vp]
        L.dart_evict_most.argtypes = [cp, ep, i32]
        L.dart_evict_workspace_bytes.argtypes = [cp, ep, i32]
        L.dart_evict_workspace_bytes.restype = sz
        L.dart_evict.argtypes = [cp, ep, vp, vp, vp, vp, vp, vp, vp, i64, vp, vp, sz, vp, vp]
        for name in ("dart_select_pivots", "dart_duplication_scores", "dart_topk_keep",
                     "dart_gather_compact", "dart_compact_sequences", "dart_reduce",
                     "dart_reduce_profiled", "dart_device_status", "dart_reduce_static",
                     "dart_device_status_static", "dart_probe_mfma_dot32",
                     "dart_score_tile_shape", "dart_score_tile_shape_first_read",
                     "dart_reduce_with_norms", "dart_norm_rotate", "dart_norm_rotate_append",
                     "dart_attend", "dart_append_4bit", "dart_read_4bit", "dart_attend_4bit",
                     "dart_attend_weights", "dart_evict"):
            getattr(L, name).restype = C.c_int
        L.dart_score_tolerance.argtypes = [i32]
        L.dart_score_tolerance.restype = C.c_double
        L.dart_strerror.argtypes = [C.c_int]
        L.dart_strerror.restype = C.c_char_p
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().dart_strerror(int(status)).decode()


def score_tolerance(dtype: int) -> float:
    return float(lib().dart_score_tolerance(int(dtype)))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    """The hipStream_t of a torch stream, of a raw handle, or of the current stream (asked for as a
    handle: a stream object costs 3 us, as much as the launch it is for)."""
    if stream is None:
        if _raw_stream is not None and _raw_device is not None:
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def make_desc(B: int, D: int, P: int, dtype: int, *, N: int = 0, K: int = 0, keep_num: int = 0,
              keep_den: int = 1, cu_seqlens: Optional[torch.Tensor] = None, total_N: int = 0,
              max_N: int = 0, ld: Optional[int] = None,
              pivot_mode: int = DART_PIVOT_MAX_L1,
              score_mode: int = DART_SCORE_PER_PIVOT,
              ext_pivots: Optional[torch.Tensor] = None, P_ext: int = 0,
              ext_ld: Optional[int] = None, span_start: Optional[torch.Tensor] = None,
              X_rows: int = 0, seed: int = 0) -> DartDesc:
    d = DartDesc()
    d.B, d.D, d.P, d.N = B, D, P, N
    d.cu_seqlens = None if cu_seqlens is None else cu_seqlens.data_ptr()
    d.total_N, d.max_N = total_N, max_N
    d.ld = D if ld is None else ld
    d.dtype, d.K, d.keep_num, d.keep_den = dtype, K, keep_num, keep_den
    d.pivot_mode, d.score_mode = pivot_mode, score_mode
    d.P_ext = P_ext
    if ext_pivots is not None:  # a tensor, or a raw device address
        d.ext_pivots = ext_pivots.data_ptr() if hasattr(ext_pivots, "data_ptr") else int(ext_pivots)
    d.ext_ld = (D if ext_ld is None else ext_ld) if P_ext > 0 else 0
    if span_start is not None:  # a tensor, or a raw device address
        d.span_start = (span_start.data_ptr() if hasattr(span_start, "data_ptr")
                        else int(span_start))
    d.X_rows = X_rows
    d.seed = seed & (2**64 - 1)
    # the descriptor holds raw device addresses: keep their tensors alive with it
    d._keepalive = (cu_seqlens, ext_pivots, span_start)
    return d


def dart_workspace_bytes(desc: DartDesc) -> int:
    return int(lib().dart_workspace_bytes(C.byref(desc)))


def alloc_workspace(desc: DartDesc, device="cuda") -> torch.Tensor:
    n = dart_workspace_bytes(desc)
    if n == 0:
        raise DartError(DART_ERR_SHAPE, "dart_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _check(status: int, where: str):
    if status != DART_OK:
        raise DartError(status, where)


def dart_select_pivots(desc, X, piv, ws, *, crit=None, crit_D=0, crit_ld=0, l1_out=None,
                       stream=None):
    _check(lib().dart_select_pivots(C.byref(desc), _ptr(X), _ptr(crit), crit_D, crit_ld,
                                    _ptr(piv), _ptr(l1_out), _ptr(ws), ws.numel(),
                                    _stream(stream)), "dart_select_pivots")


def dart_duplication_scores(desc, X, piv, S, ws, *, stream=None):
    _check(lib().dart_duplication_scores(C.byref(desc), _ptr(X), _ptr(piv), _ptr(S), _ptr(ws),
                                         ws.numel(), _stream(stream)), "dart_duplication_scores")


def dart_topk_keep(desc, S, piv, keep, ws, *, X=None, cu_keep=None, stream=None):
    _check(lib().dart_topk_keep(C.byref(desc), _ptr(S), _ptr(piv), _ptr(X), _ptr(keep),
                                _ptr(cu_keep), _ptr(ws), ws.numel(), _stream(stream)),
           "dart_topk_keep")


def dart_gather_compact(desc, X, keep, Y, ws, *, pos=None, pos_out=None, stream=None):
    _check(lib().dart_gather_compact(C.byref(desc), _ptr(X), _ptr(pos), _ptr(keep), _ptr(Y),
                                     _ptr(pos_out), _ptr(ws), ws.numel(), _stream(stream)),
           "dart_gather_compact")


def dart_compact_sequences(desc, seq_cu, keep, tensors, seq_cu_out, row_map, ws, *, pos=None,
                           pos_out=None, stream=None):
    """tensors: list of (src, dst) 2-D tensors with contiguous rows (any row stride).
    pos / pos_out: [planes, rows] int64 tensors (plane-major), or None."""
    arr = (DartRowTensor * max(len(tensors), 1))()
    for i, (src, dst) in enumerate(tensors):
        esz = src.element_size()
        arr[i] = DartRowTensor(src.data_ptr(), dst.data_ptr(), src.shape[1] * esz,
                               src.stride(0) * esz, dst.stride(0) * esz)
    planes = 0 if pos is None else pos.shape[0]
    _check(lib().dart_compact_sequences(
        C.byref(desc), _ptr(seq_cu), _ptr(keep), len(tensors), arr, _ptr(pos), planes,
        0 if pos is None else pos.stride(0), _ptr(pos_out),
        0 if pos_out is None else pos_out.stride(0), _ptr(seq_cu_out), _ptr(row_map), _ptr(ws),
        ws.numel(), _stream(stream)), "dart_compact_sequences")


def dart_reduce(desc, X, Y, keep, ws, *, crit=None, crit_D=0, crit_ld=0, pos=None, pos_out=None,
                cu_keep=None, piv_out=None, S_out=None, stream=None):
    _check(lib().dart_reduce(C.byref(desc), _ptr(X), _ptr(crit), crit_D, crit_ld, _ptr(pos),
                             _ptr(Y), _ptr(pos_out), _ptr(keep), _ptr(cu_keep), _ptr(piv_out),
                             _ptr(S_out), _ptr(ws), ws.numel(), _stream(stream)), "dart_reduce")


def dart_reduce_with_norms(desc, X, Y, keep, ws, l1, l1_rel_err, *, crit=None, crit_D=0,
                           crit_ld=0, pos=None, pos_out=None, cu_keep=None, piv_out=None,
                           S_out=None, stream=None):
    """dart_reduce without its norm pass: l1 holds the criterion norms, good to l1_rel_err."""
    _check(lib().dart_reduce_with_norms(C.byref(desc), _ptr(X), _ptr(crit), crit_D, crit_ld,
                                        _ptr(l1), float(l1_rel_err), _ptr(pos), _ptr(Y),
                                        _ptr(pos_out), _ptr(keep), _ptr(cu_keep), _ptr(piv_out),
                                        _ptr(S_out), _ptr(ws), ws.numel(), _stream(stream)),
           "dart_reduce_with_norms")


def dart_reduce_static(desc, X, Y, keep, *, crit=None, crit_D=0, crit_ld=0, pos=None,
                       pos_out=None, cu_keep=None, piv_out=None, S_out=None, stream=None):
    """dart_reduce on the library's built-in scratch buffer: no workspace, no allocation."""
    _check(lib().dart_reduce_static(C.byref(desc), _ptr(X), _ptr(crit), crit_D, crit_ld,
                                    _ptr(pos), _ptr(Y), _ptr(pos_out), _ptr(keep),
                                    _ptr(cu_keep), _ptr(piv_out), _ptr(S_out), _stream(stream)),
           "dart_reduce_static")


def dart_score_tile_shape(desc) -> tuple:
    """(waves per workgroup, groups of them) of the score kernel for this descriptor; (0, 0)
    for fp32."""
    w, ks = C.c_int32(0), C.c_int32(0)
    _check(lib().dart_score_tile_shape(C.byref(desc), C.byref(w), C.byref(ks)),
           "dart_score_tile_shape")
    return int(w.value), int(ks.value)


def dart_score_tile_shape_first_read(desc) -> tuple:
    """The same for calls whose score pass is the first pass over X (a separate criterion
    tensor, the stage entry point)."""
    w, ks = C.c_int32(0), C.c_int32(0)
    _check(lib().dart_score_tile_shape_first_read(C.byref(desc), C.byref(w), C.byref(ks)),
           "dart_score_tile_shape_first_read")
    return int(w.value), int(ks.value)


def dart_static_scratch_bytes() -> int:
    return int(lib().dart_static_scratch_bytes())


def dart_device_status_static(desc, *, stream=None) -> int:
    return int(lib().dart_device_status_static(C.byref(desc), _stream(stream)))


def dart_probe_mfma_dot32(A, B, out, *, stream=None):
    """A, B: bf16 [tiles, 16, 32]; out: float32 [tiles, 16, 16] (raw matrix-core sums)."""
    _check(lib().dart_probe_mfma_dot32(_ptr(A), _ptr(B), _ptr(out), A.shape[0], _stream(stream)),
           "dart_probe_mfma_dot32")


def dart_reduce_profiled(desc, X, Y, keep, ws, events, *, crit=None, crit_D=0, crit_ld=0,
                         pos=None, pos_out=None, cu_keep=None, piv_out=None, S_out=None,
                         stream=None):
    """events: 12 raw hipEvent_t handles (ints): begin and end of the six stages."""
    assert len(events) == 12
    arr = (C.c_void_p * 12)(*[C.c_void_p(int(e)) for e in events])
    _check(lib().dart_reduce_profiled(C.byref(desc), _ptr(X), _ptr(crit), crit_D, crit_ld,
                                      _ptr(pos), _ptr(Y), _ptr(pos_out), _ptr(keep),
                                      _ptr(cu_keep), _ptr(piv_out), _ptr(S_out), _ptr(ws),
                                      ws.numel(), _stream(stream), arr), "dart_reduce_profiled")


def dart_device_status(desc, ws, *, stream=None) -> int:
    return int(lib().dart_device_status(C.byref(desc), _ptr(ws), _stream(stream)))


# ---- attention on either side of the step ---------------------------------------------------

_DTYPES = {torch.float32: DART_F32, torch.bfloat16: DART_BF16}
_KINDS = {v: k for k, v in _DTYPES.items()}

# These calls are made once or twice per layer and token, so what they check on the way is kept to
# a few comparisons; a message is put together only for what is refused.


def _ints(t, what: str):
    """An int32 device tensor whose last dimension is contiguous."""
    if t.dtype != torch.int32 or (t.numel() > 0 and t.stride(-1) != 1):
        raise ValueError(f"{what}: int32, contiguous rows")
    return t


def _rows(t, kind, T: int, heads: int, d: int, what: str):
    """(address, row stride) of a tensor of rows [T, heads*d] or [T, heads, d] with contiguous
    rows, such as a slice of a fused projection's output."""
    shape, stride, width = t.shape, t.stride(), heads * d
    if shape == (T, width):
        good = stride[1] == 1
    else:
        good = shape == (T, heads, d) and stride[2] == 1 and (heads == 1 or stride[1] == d)
    if not good or t.dtype is not kind:
        raise ValueError(f"{what}: [{T}, {width}] of {kind} with contiguous rows")
    return t.data_ptr(), (stride[0] if T > 1 else width)


def _plain(t, T: int, n: int, what: str):
    """The address of a contiguous float32 tensor of T*n values, or None."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != T * n or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous float32, {T * n} values")
    return t.data_ptr()


def _status(t):
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() != 1:
        raise ValueError("status: int32 [1]")
    return t.data_ptr()


def _table(t):
    """(row stride, entries of a row) of a page table, which may be a view of a wider one."""
    return (t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)), t.shape[1]


def make_rotation(Hq: int, Hkv: int, d: int, dtype: int, inv_freq: torch.Tensor, *,
                  interleaved: bool = False, sections=None,
                  q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                  eps: float = 1e-6, scale: float = 1.0) -> DartRotation:
    """inv_freq: float32 [rot/2] on the device.  sections: pairs that follow each plane of position
    ids, or None for one plane."""
    r = DartRotation()
    sections = [inv_freq.numel()] if sections is None else list(sections)
    if inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq: contiguous float32")
    if not 1 <= len(sections) <= 4 or sum(sections) != inv_freq.numel():
        raise ValueError("sections: up to 4, summing to the pairs")
    for w in (q_weight, k_weight):
        if w is not None and (w.numel() != d or not w.is_contiguous() or _DTYPES.get(w.dtype) != dtype):
            raise ValueError("weights: contiguous [d] of the rows' dtype")
    r.Hq, r.Hkv, r.d, r.dtype = Hq, Hkv, d, dtype
    r.rot, r.interleaved, r.planes = 2 * inv_freq.numel(), int(interleaved), len(sections)
    r.sections[:len(sections)] = sections
    r.inv_freq = inv_freq.data_ptr()
    r.q_weight = None if q_weight is None else q_weight.data_ptr()
    r.k_weight = None if k_weight is None else k_weight.data_ptr()
    r.eps, r.scale = eps, scale
    # the descriptor holds raw device addresses: keep their tensors alive with it
    r._keepalive = (inv_freq, q_weight, k_weight)
    r._ref, r._heads = C.byref(r), (_KINDS.get(dtype), Hq, Hkv, d, len(sections))
    return r


def make_cache(Hq: int, pool: torch.Tensor, pages: torch.Tensor, kv_len: torch.Tensor, max_kv: int, *,
               T: Optional[int] = None, max_q: Optional[int] = None, cu_q: Optional[torch.Tensor] = None,
               group_cu: Optional[torch.Tensor] = None, prefix_pages: Optional[torch.Tensor] = None,
               prefix_len: Optional[torch.Tensor] = None, max_prefix: Optional[int] = None) -> DartCache:
    """pool: the key pool [pages, Hkv, page_size, d], any strides with contiguous heads (so a pool
    whose memory holds [pages, page_size, Hkv, d] is passed transposed); the value pool is laid out
    like it.  pages: int32 [B, n]; kv_len: int32 [B] with the tokens of the call.  cu_q: int32 [B+1] and T
    tokens, at most max_q of a sequence (any number by default; a bound near the truth divides the
    work better); without it one token each.  max_prefix: keys of a prefix at most (by default as many as its row of
    prefix_pages has room for)."""
    if pool.dim() != 4 or pool.stride(3) != 1 or pool.dtype not in _DTYPES:
        raise ValueError("pool: [pages, Hkv, page_size, d] with contiguous heads")
    return _cache(Hq, pool.shape[3], pool.dtype, pool, 1, pages, kv_len, max_kv, T, max_q, cu_q, group_cu, prefix_pages, prefix_len,
                  max_prefix)


def _cache(Hq, d, kind, pool, values, pages, kv_len, max_kv, T, max_q, cu_q, group_cu, prefix_pages, prefix_len, max_prefix):
    """The descriptor; values: of an element of the pool."""
    if pages.dim() != 2 or kv_len.numel() != pages.shape[0]:
        raise ValueError("pages: [B, n], kv_len: [B]")
    c = DartCache()
    c.B, c.Hq, c.Hkv, c.d, c.dtype = pages.shape[0], Hq, pool.shape[1], d, _DTYPES[kind]
    if cu_q is not None and (T is None or cu_q.numel() != c.B + 1):
        raise ValueError("cu_q: [B+1], with T")
    c.T = c.B if T is None else T
    c.max_q, c.max_kv = (1 if cu_q is None else c.T) if max_q is None else max_q, max_kv
    c.cu_q = None if cu_q is None else _ints(cu_q, "cu_q").data_ptr()
    c.kv_len, c.pages = _ints(kv_len, "kv_len").data_ptr(), _ints(pages, "pages").data_ptr()
    c.pages_ld, c.pages_n = _table(pages)
    if c.pages_n == 0:  # (a table without columns: 0 would stand for pages_ld)
        c.max_kv = 0
    c.n_pages, c.page_size = pool.shape[0], pool.shape[2]
    c.row_ld = pool.stride(2) * values if c.page_size > 1 else pool.shape[3] * values
    c.head_ld = pool.stride(1) * values if c.Hkv > 1 else 0
    c.page_ld = pool.stride(0) * values if c.n_pages > 1 else 0
    if group_cu is not None:
        c.groups = prefix_len.numel()
        if group_cu.numel() != c.groups + 1 or prefix_pages.dim() != 2 or prefix_pages.shape[0] != c.groups:
            raise ValueError("group_cu: [groups+1], prefix_pages: [groups, n], prefix_len: [groups]")
        c.group_cu, c.prefix_len = _ints(group_cu, "group_cu").data_ptr(), _ints(prefix_len, "prefix_len").data_ptr()
        c.prefix_pages = _ints(prefix_pages, "prefix_pages").data_ptr()
        c.prefix_ld, c.prefix_n = _table(prefix_pages)
        room = min(c.prefix_n * c.page_size, 1 << 27)  # (the most that is accepted)
        c.max_prefix = room if max_prefix is None else max_prefix if c.prefix_n else 0
    c._keepalive = (pages, kv_len, cu_q, group_cu, prefix_pages, prefix_len)
    c._ref, c._heads = C.byref(c), (kind, Hq, c.Hkv, c.d, c.T)
    c._pool, c._scales = (pool.shape, pool.stride()), None
    return c


def _pool(cache: DartCache, p, what: str):
    shape, stride = cache._pool
    if not isinstance(p, torch.Tensor) or p.shape != shape or p.dtype is not cache._heads[0] or (
            p.stride() != stride and any(a != b for a, b, n in zip(p.stride(), stride, shape) if n > 1)):
        raise ValueError(f"{what}: shape, strides and dtype of the pool the descriptor was made for")
    return p.data_ptr()


def _planes(pos, planes: int, T: int):
    """(address, plane stride) of position ids [T] or [planes, T] (or one plane expanded to that), int64."""
    shape, stride = pos.shape, pos.stride()
    if pos.dtype is not torch.int64 or shape[-1] != T or (T > 1 and stride[-1] != 1) or (
            shape[0] != planes if len(shape) == 2 else planes != 1):
        raise ValueError(f"pos: int64 [{planes}, {T}]")
    return pos.data_ptr(), (stride[0] if planes > 1 else 0)


def dart_norm_rotate(rotation: DartRotation, q, k, pos, q_out, k_out, *, l1_out=None, stream=None):
    """Heads of q [T, Hq*d] and k [T, Hkv*d] normed and turned by their position ids (int64 [T] or
    [planes, T]) into q_out and k_out (which may be q and k); l1_out float32 [T]: the L1 norms
    of the key rows."""
    T = q.shape[0]
    kind, Hq, Hkv, d, planes = rotation._heads
    qp, q_ld = _rows(q, kind, T, Hq, d, "q")
    kp, k_ld = _rows(k, kind, T, Hkv, d, "k")
    qo, qo_ld = _rows(q_out, kind, T, Hq, d, "q_out")
    ko, ko_ld = _rows(k_out, kind, T, Hkv, d, "k_out")
    pp, p_ld = _planes(pos, planes, T)
    l1 = _plain(l1_out, T, 1, "l1_out")
    if T == 0:
        return
    rc = (_lib or lib()).dart_norm_rotate(rotation._ref, T, qp, q_ld, kp, k_ld, pp, p_ld, qo, qo_ld, ko, ko_ld, l1,
                                          _stream(stream))
    if rc:
        _check(rc, "dart_norm_rotate")


def dart_norm_rotate_append(rotation: DartRotation, cache: DartCache, q, k, v, pos, q_out, k_pool, v_pool, *,
                            k_out=None, l1_out=None, status=None, stream=None):
    """dart_norm_rotate for the tokens of `cache`, keys and values going to their pages.  status:
    int32 [1] that bits are OR-ed into, or None."""
    kind, Hq, Hkv, d, planes = rotation._heads
    T = cache._heads[4]
    qp, q_ld = _rows(q, kind, T, Hq, d, "q")
    kp, k_ld = _rows(k, kind, T, Hkv, d, "k")
    vp, v_ld = _rows(v, kind, T, Hkv, d, "v")
    qo, qo_ld = _rows(q_out, kind, T, Hq, d, "q_out")
    ko, ko_ld = (None, 0) if k_out is None else _rows(k_out, kind, T, Hkv, d, "k_out")
    pp, p_ld = _planes(pos, planes, T)
    k_at, v_at = _pool(cache, k_pool, "k_pool"), _pool(cache, v_pool, "v_pool")
    l1, st = _plain(l1_out, T, 1, "l1_out"), _status(status)
    if T == 0:
        return
    rc = (_lib or lib()).dart_norm_rotate_append(rotation._ref, cache._ref, qp, q_ld, kp, k_ld, vp, v_ld, pp, p_ld, qo,
                                                 qo_ld, ko, ko_ld, l1, k_at, v_at, st, _stream(stream))
    if rc:
        _check(rc, "dart_norm_rotate_append")


def dart_attend_workspace_bytes(cache: DartCache) -> int:
    return int(lib().dart_attend_workspace_bytes(C.byref(cache)))


def alloc_attend_workspace(cache: DartCache, device="cuda") -> torch.Tensor:
    n = dart_attend_workspace_bytes(cache)
    if n == 0:
        raise DartError(DART_ERR_SHAPE, "dart_attend_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def dart_attend(cache: DartCache, q, k_pool, v_pool, out, ws, *, scale: float, causal: bool = True, lse=None,
                status=None, stream=None):
    """Attention of the tokens' queries q [T, Hq*d] over the cache (and the shared prefixes) into
    out [T, Hq*d]; lse float32 [T, Hq]."""
    kind, Hq, _, d, T = cache._heads
    qp, q_ld = _rows(q, kind, T, Hq, d, "q")
    o, o_ld = _rows(out, kind, T, Hq, d, "out")
    k_at, v_at = _pool(cache, k_pool, "k_pool"), _pool(cache, v_pool, "v_pool")
    le, st = _plain(lse, T, Hq, "lse"), _status(status)
    if T == 0:
        return
    rc = (_lib or lib()).dart_attend(cache._ref, qp, q_ld, k_at, v_at, scale, causal, o, o_ld, le, ws.data_ptr(),
                                     ws.numel(), st, _stream(stream))
    if rc:
        _check(rc, "dart_attend")


# ---- a cache held in 4 bits ------------------------------------------------------------------


def alloc_pool_4bit(n_pages: int, Hkv: int, page_size: int, d: int, device="cuda"):
    """A pool held in 4 bits, all zeros: (codes, scales), uint8 [n_pages, Hkv, page_size, 16 or 1 times the blocks of
    32 values in a head]."""
    blocks = -(-d // 32)
    return tuple(torch.zeros((n_pages, Hkv, page_size, blocks * n), dtype=torch.uint8, device=device) for n in (16, 1))


def make_cache_4bit(Hq: int, d: int, dtype: int, pool, pages: torch.Tensor, kv_len: torch.Tensor, max_kv: int, *,
                    T: Optional[int] = None, max_q: Optional[int] = None, cu_q: Optional[torch.Tensor] = None,
                    group_cu: Optional[torch.Tensor] = None, prefix_pages: Optional[torch.Tensor] = None,
                    prefix_len: Optional[torch.Tensor] = None, max_prefix: Optional[int] = None) -> DartCache:
    """make_cache for pools held in 4 bits.  pool: (codes, scales) as alloc_pool_4bit makes them, any strides with contiguous
    heads that are alike for both (a pool whose memory holds [pages, page_size, Hkv, ...] is passed transposed);
    d, dtype: elements of a head and dtype of the rows."""
    codes, scales = pool
    blocks = -(-d // 32)
    if codes.dim() != 4 or codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or dtype not in _KINDS or (
            codes.shape != (*scales.shape[:3], 16 * blocks)) or scales.shape[3] != blocks or codes.stride(3) != 1 or (
            blocks > 1 and scales.stride(3) != 1) or any(
            n > 1 and x != 16 * y for n, x, y in zip(codes.shape[:3], codes.stride(), scales.stride())):
        raise ValueError(f"pool: uint8 codes [pages, Hkv, page_size, {16 * blocks}] and scales [..., {blocks}], heads contiguous, "
                         "strides alike")
    c = _cache(Hq, d, _KINDS[dtype], codes, 2, pages, kv_len, max_kv, T, max_q, cu_q, group_cu, prefix_pages, prefix_len, max_prefix)
    c._scales = (scales.shape, scales.stride())
    return c


def _alike(t, like) -> bool:
    """uint8, of this shape and strides (where they count)."""
    shape, stride = like
    return t.dtype is torch.uint8 and t.shape == shape and (
        t.stride() == stride or all(a == b for a, b, n in zip(t.stride(), stride, shape) if n > 1))


def _codes(cache: DartCache, p, what: str):
    """Addresses of (codes, scales)."""
    if cache._scales is None:
        raise ValueError("cache: of make_cache_4bit")
    if not isinstance(p, (tuple, list)) or len(p) != 2 or not _alike(p[0], cache._pool) or not _alike(p[1], cache._scales):
        raise ValueError(f"{what}: (codes, scales) as of the pool the descriptor was made for")
    return p[0].data_ptr(), p[1].data_ptr()


def _held(cache: DartCache, p, what: str):
    """Addresses of (codes, scales), or of a pool of rows and None."""
    return (_pool(cache, p, what), None) if cache._scales is None else _codes(cache, p, what)


def _workspace(n: int, where: str, device):
    if n == 0:
        raise DartError(DART_ERR_SHAPE, where)
    return torch.empty(n, dtype=torch.uint8, device=device)


def dart_append_4bit(cache: DartCache, k, v, k_pool, v_pool, *, status=None, stream=None):
    """Key and value rows [T, Hkv*d] of the cache's tokens to their places in pages held in 4 bits."""
    kind, _, Hkv, d, T = cache._heads
    kp, k_ld = _rows(k, kind, T, Hkv, d, "k")
    vp, v_ld = _rows(v, kind, T, Hkv, d, "v")
    kc, ks = _codes(cache, k_pool, "k_pool")
    vc, vs = _codes(cache, v_pool, "v_pool")
    st = _status(status)
    if T == 0:
        return
    rc = (_lib or lib()).dart_append_4bit(cache._ref, kp, k_ld, vp, v_ld, kc, ks, vc, vs, st, _stream(stream))
    if rc:
        _check(rc, "dart_append_4bit")


def dart_read_4bit(cache: DartCache, k_pool, v_pool, k_out=None, v_out=None, *, status=None, stream=None):
    """The rows [T, Hkv*d] of the cache's tokens as the pages hold them into k_out and v_out (either may be None)."""
    kind, _, Hkv, d, T = cache._heads
    ko, k_ld = (None, 0) if k_out is None else _rows(k_out, kind, T, Hkv, d, "k_out")
    vo, v_ld = (None, 0) if v_out is None else _rows(v_out, kind, T, Hkv, d, "v_out")
    kc, ks = (None, None) if k_out is None else _codes(cache, k_pool, "k_pool")
    vc, vs = (None, None) if v_out is None else _codes(cache, v_pool, "v_pool")
    st = _status(status)
    if T == 0:
        return
    rc = (_lib or lib()).dart_read_4bit(cache._ref, kc, ks, vc, vs, ko, k_ld, vo, v_ld, st, _stream(stream))
    if rc:
        _check(rc, "dart_read_4bit")


def dart_attend_4bit_workspace_bytes(cache: DartCache) -> int:
    return int(lib().dart_attend_4bit_workspace_bytes(C.byref(cache)))


def alloc_attend_4bit_workspace(cache: DartCache, device="cuda") -> torch.Tensor:
    return _workspace(dart_attend_4bit_workspace_bytes(cache), "dart_attend_4bit_workspace_bytes", device)


def dart_attend_4bit(cache: DartCache, q, k_pool, v_pool, out, ws, *, scale: float, causal: bool = True, lse=None,
                     status=None, stream=None):
    """dart_attend over pools held in 4 bits."""
    kind, Hq, _, d, T = cache._heads
    qp, q_ld = _rows(q, kind, T, Hq, d, "q")
    o, o_ld = _rows(out, kind, T, Hq, d, "out")
    kc, ks = _codes(cache, k_pool, "k_pool")
    vc, vs = _codes(cache, v_pool, "v_pool")
    le, st = _plain(lse, T, Hq, "lse"), _status(status)
    if T == 0:
        return
    rc = (_lib or lib()).dart_attend_4bit(cache._ref, qp, q_ld, kc, ks, vc, vs, scale, causal, o, o_ld, le, ws.data_ptr(),
                                          ws.numel(), st, _stream(stream))
    if rc:
        _check(rc, "dart_attend_4bit")


# ---- eviction ---------------------------------------------------------------------------------


def _gathered(cache: DartCache, w, what: str):
    """The address of the weights of a cache's keys: contiguous float32 [pages, Hkv, page_size]."""
    if w.dtype is not torch.float32 or w.shape != cache._pool[0][:3] or not w.is_contiguous():
        raise ValueError(f"{what}: contiguous float32 {tuple(cache._pool[0][:3])}")
    return w.data_ptr()


def dart_attend_weights_workspace_bytes(cache: DartCache) -> int:
    return int(lib().dart_attend_weights_workspace_bytes(C.byref(cache), cache._scales is not None))


def alloc_attend_weights_workspace(cache: DartCache, device="cuda") -> torch.Tensor:
    return _workspace(dart_attend_weights_workspace_bytes(cache), "dart_attend_weights_workspace_bytes", device)


def dart_attend_weights(cache: DartCache, q, k_pool, lse, weights, ws, *, scale: float, causal: bool = True, carry: float = 1.0,
                        status=None, stream=None):
    """weights (float32 [pages, Hkv, page_size]) of every key: carry times what they were, and what the tokens' queries
    q [T, Hq*d] with the lse [T, Hq] of dart_attend give it.  Keys of the call's tokens start from 0.  k_pool: rows, or (codes, scales)
    of a cache of make_cache_4bit."""
    kind, Hq, _, d, T = cache._heads
    qp, q_ld = _rows(q, kind, T, Hq, d, "q")
    kp, ks = _held(cache, k_pool, "k_pool")
    if lse is None:
        raise ValueError("lse: as of dart_attend")
    le, w, st = _plain(lse, T, Hq, "lse"), _gathered(cache, weights, "weights"), _status(status)
    if T == 0:
        return
    rc = (_lib or lib()).dart_attend_weights(cache._ref, qp, q_ld, kp, ks, le, scale, causal, carry, w, ws.data_ptr(), ws.numel(),
                                             st, _stream(stream))
    if rc:
        _check(rc, "dart_attend_weights")


def make_eviction(*, budget: int = 0, ratio=None, first: int = 0, recent: int = 0) -> DartEviction:
    """Keys that a sequence keeps: `budget`, or where that is 0 ratio[0]/ratio[1] of its keys; the first and the recent ones
    always."""
    if budget == 0 and ratio is None:
        raise ValueError("budget or ratio")
    e = DartEviction()
    e.budget, (e.ratio_num, e.ratio_den), e.first, e.recent = budget, ratio or (0, 1), first, recent
    e._ref = C.byref(e)
    return e


def dart_evict_most(cache: DartCache, eviction: DartEviction) -> int:
    """Keys that a sequence keeps at most (entries of a row of `kept`)."""
    n = int(lib().dart_evict_most(C.byref(cache), C.byref(eviction), cache._scales is not None))
    if n < 0:
        raise DartError(DART_ERR_SHAPE, "dart_evict_most")
    return n


def dart_evict_workspace_bytes(cache: DartCache, eviction: DartEviction) -> int:
    return int(lib().dart_evict_workspace_bytes(C.byref(cache), C.byref(eviction), cache._scales is not None))


def alloc_evict_workspace(cache: DartCache, eviction: DartEviction, device="cuda") -> torch.Tensor:
    return _workspace(dart_evict_workspace_bytes(cache, eviction), "dart_evict_workspace_bytes", device)


def dart_evict(cache: DartCache, eviction: DartEviction, k_pool, v_pool, weights, kv_len_out, ws, *, weights_out=None, kept=None,
               status=None, stream=None):
    """Every sequence cut to the keys of largest weight, moved to the front of its pages; kv_len_out int32 [B] (may be the
    kv_len of the cache), weights_out like weights (may be weights), kept int32 [B, Hkv, n]: the places they had."""
    kp, ks = _held(cache, k_pool, "k_pool")
    vp, vs = _held(cache, v_pool, "v_pool")
    w, w_out = _gathered(cache, weights, "weights"), None if weights_out is None else _gathered(cache, weights_out, "weights_out")
    if kv_len_out.dtype is not torch.int32 or kv_len_out.numel() != cache.B or not kv_len_out.is_contiguous():
        raise ValueError(f"kv_len_out: contiguous int32 [{cache.B}]")
    at, ld = None, 0
    if kept is not None:
        if kept.dtype is not torch.int32 or kept.dim() != 3 or kept.shape[:2] != (cache.B, cache.Hkv) or not kept.is_contiguous():
            raise ValueError(f"kept: contiguous int32 [{cache.B}, {cache.Hkv}, n]")
        at, ld = kept.data_ptr(), kept.shape[2]
    st = _status(status)
    if cache.B == 0:
        return
    rc = (_lib or lib()).dart_evict(cache._ref, eviction._ref, kp, ks, vp, vs, w, w_out, at, ld, kv_len_out.data_ptr(), ws.data_ptr(),
                                    ws.numel(), st, _stream(stream))
    if rc:
        _check(rc, "dart_evict")
