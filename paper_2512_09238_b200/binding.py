"""ctypes binding of the C-ABI library declared in ``include/tca.h``.

Argument marshalling only: every function below has the name and the argument order of
its C counterpart, takes torch CUDA tensors (device buffers) or numpy arrays (host
buffers), passes raw pointers and sizes, and raises :class:`TcaError` on a non-zero
status.  Nothing is computed in Python and nothing falls back to the CPU: if
``libtca.so`` has not been built, importing the library handle raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtca.so")

TCA_OK, TCA_ERR_INVALID_ARG, TCA_ERR_UNSUPPORTED, TCA_ERR_WORKSPACE = 0, -1, -2, -3
TCA_ERR_CUDA, TCA_ERR_TIMEOUT, TCA_ERR_CAPACITY, TCA_ERR_SCRATCH_LIMIT, TCA_ERR_BOUNDS = -4, -5, -6, -7, -8
TCA_DECODE_STATIC_SCRATCH_BYTES = 16 << 20
TCA_F32, TCA_BF16 = 0, 1
TCA_FLAG_PREFILL_SIMT, TCA_FLAG_ENTROPY_INDEX, TCA_FLAG_RANDOM_ORDER, TCA_FLAG_FLAT_TOPB = 1, 2, 4, 8
TCA_FLAG_PREFILL_BAND_FIRST = 16
TCA_BUILD_DEBUG_BOUNDS = 1
(TCA_OP_SCORE, TCA_OP_SELECT, TCA_OP_COMPACT, TCA_OP_PREFILL, TCA_OP_DECODE, TCA_OP_APPEND, TCA_OP_CALIB,
 TCA_OP_SCORE_SELECT, TCA_OP_PACKED) = range(9)
TCA_TREE_MAX = 128
TCA_STATE_WORDS = 8
TCA_PG_STATE_WORDS = 4
TCA_PG_LEN, TCA_PG_NEXT, TCA_PG_CHECK = 0, 1, 2

EXPORTS = (
    "tca_strerror", "tca_version", "tca_budget_resolve", "tca_workspace_bytes", "tca_score",
    "tca_select", "tca_cache_init", "tca_compact_kv", "tca_attn_prefill", "tca_attn_decode",
    "tca_cache_append", "tca_ws_status", "tca_attn_decode_static", "tca_attn_prefill_rows",
    "tca_calib_colmean", "tca_calib_score", "tca_calib_choose", "tca_calib_candidates",
    "tca_decode_static_status", "tca_selftest_wait_expiry", "tca_score_select", "tca_build_info",
    "tca_cache_status", "tca_attn_prefill_gather", "tca_compact_kv_range",
    "tca_attn_packed", "tca_cache_load", "tca_attn_tree", "tca_attn_tree_workspace_bytes", "tca_cache_accept",
    "tca_attn_window", "tca_paged_append", "tca_attn_paged", "tca_attn_paged_workspace_bytes", "tca_paged_evict",
    "tca_paged_status",
)


class TcaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().tca_strerror(status).decode()} ({status})")


class tca_params(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("block", C.c_int32), ("window", C.c_int32),
                ("alpha", C.c_float), ("sm_scale", C.c_float), ("dtype", C.c_int32),
                ("flags", C.c_int32), ("seed", C.c_int32)]


class tca_cache_desc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pos", C.c_void_p), ("state", C.c_void_p),
                ("rows_total", C.c_int64), ("n_units", C.c_int64), ("tail_cap", C.c_int64),
                ("seg_start", C.c_void_p), ("global_cap", C.c_void_p), ("n_global", C.c_void_p),
                ("tail_head", C.c_void_p), ("n_tail", C.c_void_p), ("seq_len", C.c_void_p),
                ("t_keep", C.c_void_p)]


class tca_paged_desc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pos", C.c_void_p), ("mass", C.c_void_p), ("table", C.c_void_p),
                ("state", C.c_void_p), ("n_pages", C.c_int64), ("n_units", C.c_int64), ("page_size", C.c_int32),
                ("max_pages", C.c_int32)]


_lib = None


def load_library(path: str) -> C.CDLL:
    """Load a build of the library from `path` and declare the argument types of its entry points."""
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with "
                           "`python -m paper_2512_09238_b200._build` (needs nvcc)")
    L = C.CDLL(path)
    L.tca_strerror.restype = C.c_char_p
    L.tca_strerror.argtypes = [C.c_int]
    L.tca_version.restype = C.c_int
    L.tca_workspace_bytes.restype = C.c_size_t
    L.tca_workspace_bytes.argtypes = [C.POINTER(tca_params), C.c_int64, C.c_int]
    L.tca_budget_resolve.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int64, C.c_void_p,
                                     C.c_void_p, C.c_void_p]
    P = C.POINTER(tca_params)
    D = C.POINTER(tca_cache_desc)
    vp, i64, sz = C.c_void_p, C.c_int64, C.c_size_t
    L.tca_score.argtypes = [P, vp, vp, i64, vp, vp, sz, vp]
    L.tca_select.argtypes = [P, vp, i64, vp, C.c_int32, vp, vp, vp, vp, vp, sz, vp]
    L.tca_score_select.argtypes = [P, vp, vp, i64, vp, C.c_int32, vp, vp, vp, vp, vp, vp, sz, vp]
    L.tca_cache_init.argtypes = [P, D, vp]
    L.tca_compact_kv.argtypes = [P, vp, vp, i64, vp, vp, vp, D, vp]
    L.tca_compact_kv_range.argtypes = [P, vp, vp, i64, i64, i64, vp, vp, vp, D, vp]
    L.tca_attn_prefill.argtypes = [P, vp, vp, vp, i64, D, vp, vp, sz, vp]
    L.tca_attn_prefill_rows.argtypes = [P, vp, vp, vp, i64, i64, i64, D, vp, vp, sz, vp]
    L.tca_attn_prefill_gather.argtypes = [P, vp, vp, vp, i64, i64, i64, vp, vp, vp, vp, sz, vp]
    L.tca_attn_packed.argtypes = [P, vp, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    L.tca_cache_load.argtypes = [P, vp, vp, i64, vp, vp, vp, C.c_int32, D, vp]
    L.tca_attn_tree.argtypes = [P, vp, vp, vp, C.c_int32, vp, vp, D, vp, vp, sz, vp]
    L.tca_attn_tree_workspace_bytes.restype = sz
    L.tca_attn_tree_workspace_bytes.argtypes = [P, C.c_int32]
    L.tca_cache_accept.argtypes = [P, D, vp, vp, vp, C.c_int32, vp, vp, vp]
    G = C.POINTER(tca_paged_desc)
    L.tca_attn_window.argtypes = [P, vp, vp, vp, i64, vp, vp, C.c_int32, vp, vp, sz, vp]
    L.tca_paged_append.argtypes = [P, vp, vp, i64, vp, vp, vp, C.c_int32, vp, G, vp]
    L.tca_attn_paged.argtypes = [P, vp, G, C.c_int32, C.c_int32, vp, vp, sz, vp]
    L.tca_attn_paged_workspace_bytes.restype = sz
    L.tca_attn_paged_workspace_bytes.argtypes = [P, G, C.c_int32]
    L.tca_paged_evict.argtypes = [P, G, C.c_int32, C.c_int32, vp, vp]
    L.tca_paged_status.argtypes = [G, vp, vp]
    L.tca_calib_colmean.argtypes = [P, vp, vp, i64, vp, vp, sz, vp]
    L.tca_calib_score.argtypes = [P, vp, i64, vp, vp, vp, vp]
    L.tca_calib_choose.argtypes = [vp, vp, C.c_int, C.c_double]
    L.tca_calib_candidates.argtypes = [C.c_int, C.c_int, C.c_double, vp]
    L.tca_attn_decode.argtypes = [P, vp, D, vp, vp, sz, vp]
    L.tca_cache_append.argtypes = [P, D, vp, vp, vp, vp]
    L.tca_ws_status.argtypes = [vp, vp]
    L.tca_cache_status.argtypes = [D, vp, vp]
    L.tca_attn_decode_static.argtypes = [P, vp, D, vp, vp]
    L.tca_decode_static_status.argtypes = [vp]
    L.tca_selftest_wait_expiry.argtypes = [vp, C.c_uint64, vp, vp]
    L.tca_build_info.argtypes = []
    for name in EXPORTS:
        if name not in ("tca_strerror", "tca_workspace_bytes", "tca_attn_tree_workspace_bytes",
                        "tca_attn_paged_workspace_bytes"):
            getattr(L, name).restype = C.c_int
    return L


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        # TCA_LIBRARY names another build of the same library, e.g. the range-checked libtca_dbg.so
        _lib = load_library(os.environ.get("TCA_LIBRARY") or LIB_PATH)
    return _lib


# ----------------------------------------------------------------------------- helpers
def make_params(batch, n_q_heads, n_kv_heads, head_dim, block, window, alpha=0.5, sm_scale=None,
                dtype=TCA_BF16, flags=0, seed=0) -> tca_params:
    if sm_scale is None:
        sm_scale = 1.0 / float(np.sqrt(head_dim))
    return tca_params(batch, n_q_heads, n_kv_heads, head_dim, block, window, alpha, sm_scale, dtype, flags, seed)


def _dev(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device buffers must be contiguous CUDA tensors")
    return t.data_ptr()


def _host(a: Optional[np.ndarray], dtype) -> Optional[int]:
    if a is None:
        return None
    if a.dtype != dtype or not a.flags["C_CONTIGUOUS"]:
        raise ValueError(f"host buffer must be a C-contiguous {np.dtype(dtype).name} array")
    return a.__array_interface__["data"][0]


# The current stream's handle without building a Stream object (0.1 us against 3.3 us per call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return (stream or torch.cuda.current_stream()).cuda_stream


def _check(status: int, where: str) -> None:
    if status != TCA_OK:
        raise TcaError(status, where)


def _ws_args(ws: Optional[torch.Tensor]):
    return (_dev(ws), 0 if ws is None else ws.numel() * ws.element_size())


def alloc_workspace(prm: tca_params, L: int, op: int, device="cuda") -> torch.Tensor:
    """A zero-filled device buffer of tca_workspace_bytes(prm, L, op) bytes (torch owns the
    memory).  Zero-filled because the first word of the prefill and decode workspaces is a
    sticky error flag that tca_ws_status reads."""
    n = tca_workspace_bytes(prm, L, op)
    if n == 0:
        raise TcaError(TCA_ERR_INVALID_ARG, "tca_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


# ----------------------------------------------------------------------------- the C entry points
def tca_version() -> int:
    return lib().tca_version()


def tca_strerror(status: int) -> str:
    return lib().tca_strerror(status).decode()


def tca_workspace_bytes(prm: tca_params, L: int, op: int) -> int:
    return int(lib().tca_workspace_bytes(C.byref(prm), L, op))


def tca_budget_resolve(p: np.ndarray, m: int):
    """p [Hkv, nK] float64 -> (n_k [Hkv, nK] int32, n_sel [Hkv] int64, tbar [Hkv] int32)."""
    p = np.ascontiguousarray(p, dtype=np.float64)
    H, nK = p.shape
    n_k = np.zeros((H, nK), dtype=np.int32)
    n_sel = np.zeros(H, dtype=np.int64)
    tbar = np.zeros(H, dtype=np.int32)
    _check(lib().tca_budget_resolve(p.ctypes.data, H, nK, m, n_k.ctypes.data, n_sel.ctypes.data,
                                    tbar.ctypes.data), "tca_budget_resolve")
    return n_k, n_sel, tbar


def tca_score(prm, q_last, K, L, logscore, ws, stream=None) -> None:
    _check(lib().tca_score(C.byref(prm), _dev(q_last), _dev(K), L, _dev(logscore), *_ws_args(ws),
                           _stream(stream)), "tca_score")


def tca_select(prm, logscore, L, n_k, idx, offsets_dev, h_out, t_out, ws, stream=None) -> None:
    n_k = np.ascontiguousarray(n_k, dtype=np.int32)
    _check(lib().tca_select(C.byref(prm), _dev(logscore), L, _host(n_k, np.int32), n_k.shape[1], _dev(idx),
                            _dev(offsets_dev), _dev(h_out), _dev(t_out), *_ws_args(ws), _stream(stream)),
           "tca_select")


def tca_score_select(prm, q_last, K, L, n_k, logscore, idx, offsets_dev, h_out, t_out, ws, stream=None) -> None:
    n_k = np.ascontiguousarray(n_k, dtype=np.int32)
    _check(lib().tca_score_select(C.byref(prm), _dev(q_last), _dev(K), L, _host(n_k, np.int32), n_k.shape[1],
                                  _dev(logscore), _dev(idx), _dev(offsets_dev), _dev(h_out), _dev(t_out),
                                  *_ws_args(ws), _stream(stream)), "tca_score_select")


def tca_build_info() -> int:
    return lib().tca_build_info()


def tca_cache_status(cache: "Cache", stream=None):
    """(status, detail) with detail = [unit, which check, offending value] when status is TCA_ERR_BOUNDS."""
    detail = np.zeros(3, dtype=np.int64)
    st = lib().tca_cache_status(C.byref(cache.desc), _stream(stream), detail.ctypes.data)
    return st, detail


def tca_cache_init(prm, cache: "Cache", stream=None) -> None:
    _check(lib().tca_cache_init(C.byref(prm), C.byref(cache.desc), _stream(stream)), "tca_cache_init")


def tca_compact_kv(prm, K, V, L, idx, offsets_dev, offsets_host, cache: "Cache", stream=None) -> None:
    _check(lib().tca_compact_kv(C.byref(prm), _dev(K), _dev(V), L, _dev(idx), _dev(offsets_dev),
                                _host(offsets_host, np.int64), C.byref(cache.desc), _stream(stream)),
           "tca_compact_kv")


def tca_compact_kv_range(prm, K, V, L, pos_begin, pos_end, idx, offsets_dev, offsets_host, cache: "Cache",
                         stream=None) -> None:
    _check(lib().tca_compact_kv_range(C.byref(prm), _dev(K), _dev(V), L, pos_begin, pos_end, _dev(idx),
                                      _dev(offsets_dev), _host(offsets_host, np.int64), C.byref(cache.desc),
                                      _stream(stream)), "tca_compact_kv_range")


def tca_attn_prefill(prm, Q, K, V, L, cache: "Cache", O, ws, stream=None) -> None:
    _check(lib().tca_attn_prefill(C.byref(prm), _dev(Q), _dev(K), _dev(V), L, C.byref(cache.desc), _dev(O),
                                  *_ws_args(ws), _stream(stream)), "tca_attn_prefill")


def tca_attn_prefill_rows(prm, Q, K, V, L, row_begin, row_end, cache: "Cache", O, ws, stream=None) -> None:
    _check(lib().tca_attn_prefill_rows(C.byref(prm), _dev(Q), _dev(K), _dev(V), L, row_begin, row_end,
                                       C.byref(cache.desc), _dev(O), *_ws_args(ws), _stream(stream)),
           "tca_attn_prefill_rows")


def tca_attn_prefill_gather(prm, Q, K, V, L, row_begin, row_end, idx, offsets_dev, O, ws, stream=None) -> None:
    _check(lib().tca_attn_prefill_gather(C.byref(prm), _dev(Q), _dev(K), _dev(V), L, row_begin, row_end,
                                         _dev(idx), _dev(offsets_dev), _dev(O), *_ws_args(ws), _stream(stream)),
           "tca_attn_prefill_gather")


def tca_attn_decode(prm, q, cache: "Cache", O, ws, stream=None) -> None:
    _check(lib().tca_attn_decode(C.byref(prm), _dev(q), C.byref(cache.desc), _dev(O), *_ws_args(ws),
                                 _stream(stream)), "tca_attn_decode")


def tca_attn_decode_static(prm, q, cache: "Cache", O, stream=None) -> None:
    """tca_attn_decode without a workspace: the partials live in a 16 MiB array inside the
    library, so the call allocates nothing.  For callers that cannot allocate device memory
    (all of it owned by a host engine's pool, or no allocator available in a latency-critical
    loop).  Calls share that array: do not let two of them overlap on the GPU."""
    _check(lib().tca_attn_decode_static(C.byref(prm), _dev(q), C.byref(cache.desc), _dev(O), _stream(stream)),
           "tca_attn_decode_static")


def tca_decode_static_status(stream=None) -> int:
    """TCA_OK, or TCA_ERR_TIMEOUT if a bounded wait gave up inside a tca_attn_decode_static call on
    this device since the last query (the array's status word and counters are then cleared)."""
    return lib().tca_decode_static_status(_stream(stream))


def tca_selftest_wait_expiry(ws, limit_ns: int, waited_ns=None, stream=None) -> None:
    """Makes one bounded device-side wait run out after limit_ns and leave through the kernels'
    abort path; afterwards tca_ws_status(ws) is TCA_ERR_TIMEOUT."""
    _check(lib().tca_selftest_wait_expiry(_dev(ws), int(limit_ns), _dev(waited_ns), _stream(stream)),
           "tca_selftest_wait_expiry")


def tca_cache_append(prm, cache: "Cache", k_new, v_new, q_cur, stream=None) -> None:
    _check(lib().tca_cache_append(C.byref(prm), C.byref(cache.desc), _dev(k_new), _dev(v_new), _dev(q_cur),
                                  _stream(stream)), "tca_cache_append")


def tca_ws_status(ws, stream=None) -> int:
    return lib().tca_ws_status(_dev(ws), _stream(stream))


_ELT = {TCA_BF16: torch.bfloat16, TCA_F32: torch.float32}
_pack4, _pack8 = struct.Struct("=4q").pack, struct.Struct("=8q").pack
_I32, _I64, _U8, _F32 = torch.int32, torch.int64, torch.uint8, torch.float32


# Without the lazy initialisation of torch.cuda.current_device(): asked only when a tensor is on a device.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_on(here: int, stream) -> int:
    """_stream for a call whose tensors are on device `here`, the current one."""
    return _raw_stream(here) if stream is None and _raw_stream is not None else _stream(stream)


def _refuse(where: str, *specs) -> None:
    """Says which argument of a serving call is wrong: specs are (name, tensor, dtype, shape, contiguous)."""
    here = torch.cuda.current_device() if torch.cuda.is_available() else -2
    for name, t, dtype, shape, whole in specs:
        if t is None and name in ("n_live", "mass"):
            continue
        if not isinstance(t, torch.Tensor) or t.get_device() != here:
            raise ValueError(f"{where}: {name} must be a tensor on the current CUDA device")
        if t.dtype != dtype or (shape is not None and t.shape != shape):
            raise ValueError(f"{where}: {name} must be {dtype} of shape {tuple(shape or t.shape)}, got {t.dtype} {tuple(t.shape)}")
        if (not t.is_contiguous()) if whole else (t.stride(-1) != 1 and t.numel() > 0):
            raise ValueError(f"{where}: {name} must be contiguous" + ("" if whole else " in its last dimension"))
    raise ValueError(f"{where}: bad argument")


# What is no tensor at all has none of the attributes that the checks below ask for: the calls catch that, which
# costs nothing otherwise, and leave it to _refuse to say which argument it is.
def _ok(t, here, dtype, shape) -> bool:
    """A contiguous tensor of this type and shape on device `here`."""
    return t.dtype is dtype and t.shape == shape and t.get_device() == here and t.is_contiguous()


def _strides(t, here, dtype, shape):
    """Element strides (head, row) of a [heads, rows, d] view of this type and shape on device `here`, with any
    strides but the last (a dimension of one element counts as contiguous: torch leaves its stride unspecified);
    None if it is not one."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != here:
        return None
    head, row, last = t.stride()
    heads, rows, d = shape
    if last != 1 and rows:
        return None
    if heads < 2 or rows < 2:
        return (head if heads > 1 else max(rows, 1) * d, row if rows > 1 else d)
    return head, row


def _host_in(where: str, name: str, a, dtype, n: int):
    """The bytes of a host array of n elements that a call only reads (a copy is cheaper than asking numpy for the
    address)."""
    if not isinstance(a, np.ndarray) or a.dtype != dtype or a.shape != (n,) or not a.flags.c_contiguous:
        raise ValueError(f"{where}: {name} must be a C-contiguous {np.dtype(dtype).name} array of {n} elements")
    return a.tobytes()


def _fits(cache: "Cache", here, dtype, d) -> bool:
    """The cache lies on device `here` and was made for this type and head size."""
    return cache.k.dtype is dtype and cache.k.shape[1] == d and cache.k.get_device() == here


def _refuse_cache(where: str, prm, cache: "Cache", *specs) -> None:
    e, here = _ELT.get(prm.dtype), torch.cuda.current_device() if torch.cuda.is_available() else -2
    if not isinstance(cache, Cache) or not _fits(cache, here, e, prm.head_dim):
        raise ValueError(f"{where}: the cache must be on the current CUDA device and made for {e} and head size {prm.head_dim}")
    _refuse(where, *specs)


def tca_attn_packed(prm, Q, K, V, rows, seq_start, O, ws, stream=None) -> None:
    """Q, O [n_q_heads, rows, d], K, V [n_kv_heads, rows, d]: contiguous, or views with any head and row strides
    that are multiples of 16 bytes (``x.transpose(0, 1)`` of a token-major tensor); seq_start a CUDA int64 tensor
    of prm.batch + 1 elements."""
    e, d = _ELT.get(prm.dtype), prm.head_dim
    qs, ks, ss = (prm.n_q_heads, rows, d), (prm.n_kv_heads, rows, d), (prm.batch + 1,)
    try:
        here = Q.get_device()
        good = (here >= 0 and here == _current_device() and (sq := _strides(Q, here, e, qs)) and (sk := _strides(K, here, e, ks))
                and (sv := _strides(V, here, e, ks)) and (so := _strides(O, here, e, qs)) and _ok(seq_start, here, _I64, ss)
                and _ok(ws, here, _U8, ws.shape))
    except AttributeError:
        good = False
    if not good:
        _refuse("tca_attn_packed", ("Q", Q, e, qs, False), ("K", K, e, ks, False), ("V", V, e, ks, False),
                ("O", O, e, qs, False), ("seq_start", seq_start, _I64, ss, True), ("ws", ws, _U8, None, True))
    _check(lib().tca_attn_packed(C.byref(prm), Q.data_ptr(), K.data_ptr(), V.data_ptr(), rows, seq_start.data_ptr(),
                                 _pack8(*sq, *sk, *sv, *so), O.data_ptr(), ws.data_ptr(), ws.numel(), _stream_on(here, stream)),
           "tca_attn_packed")


def tca_attn_window(prm, Q, K, V, rows, seq_start, n_sink, O, ws, stream=None) -> None:
    """tca_attn_packed with a sliding window of prm.window keys and the first n_sink keys of each sequence always
    visible; buffers and workspace (TCA_OP_PACKED) as there."""
    e, d = _ELT.get(prm.dtype), prm.head_dim
    qs, ks, ss = (prm.n_q_heads, rows, d), (prm.n_kv_heads, rows, d), (prm.batch + 1,)
    try:
        here = Q.get_device()
        good = (here >= 0 and here == _current_device() and (sq := _strides(Q, here, e, qs)) and (sk := _strides(K, here, e, ks))
                and (sv := _strides(V, here, e, ks)) and (so := _strides(O, here, e, qs)) and _ok(seq_start, here, _I64, ss)
                and _ok(ws, here, _U8, ws.shape))
    except AttributeError:
        good = False
    if not good:
        _refuse("tca_attn_window", ("Q", Q, e, qs, False), ("K", K, e, ks, False), ("V", V, e, ks, False),
                ("O", O, e, qs, False), ("seq_start", seq_start, _I64, ss, True), ("ws", ws, _U8, None, True))
    _check(lib().tca_attn_window(C.byref(prm), Q.data_ptr(), K.data_ptr(), V.data_ptr(), rows, seq_start.data_ptr(),
                                 _pack8(*sq, *sk, *sv, *so), n_sink, O.data_ptr(), ws.data_ptr(), ws.numel(), _stream_on(here, stream)),
           "tca_attn_window")


def tca_cache_load(prm, K, V, rows, seq_start, slots, cache: "Cache", stream=None) -> None:
    """K, V [n_kv_heads, rows, d] as in tca_attn_packed; seq_start an int64 and slots an int32 numpy array (or None)."""
    e, ks = _ELT.get(prm.dtype), (prm.n_kv_heads, rows, prm.head_dim)
    try:
        here = K.get_device()
        good = (here >= 0 and here == _current_device() and (sk := _strides(K, here, e, ks)) and (sv := _strides(V, here, e, ks))
                and _fits(cache, here, e, prm.head_dim))
    except AttributeError:
        good = False
    if not good:
        _refuse_cache("tca_cache_load", prm, cache, ("K", K, e, ks, False), ("V", V, e, ks, False))
    n_seq = len(seq_start) - 1 if isinstance(seq_start, np.ndarray) and seq_start.ndim == 1 else -1
    starts = _host_in("tca_cache_load", "seq_start", seq_start, np.int64, n_seq + 1)
    places = None if slots is None else _host_in("tca_cache_load", "slots", slots, np.int32, n_seq)
    _check(lib().tca_cache_load(C.byref(prm), K.data_ptr(), V.data_ptr(), rows, _pack4(*sk, *sv),
                                starts, places, n_seq, C.byref(cache.desc),
                                _stream_on(here, stream)), "tca_cache_load")


def tca_attn_tree_workspace_bytes(prm, n_draft: int) -> int:
    return int(lib().tca_attn_tree_workspace_bytes(C.byref(prm), n_draft))


def alloc_tree_workspace(prm: tca_params, n_draft: int, device="cuda") -> torch.Tensor:
    """A zero-filled workspace for tca_attn_tree calls of n_draft drafted tokens."""
    n = tca_attn_tree_workspace_bytes(prm, n_draft)
    if n == 0:
        raise TcaError(TCA_ERR_INVALID_ARG, "tca_attn_tree_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def tca_attn_tree(prm, q, k_draft, v_draft, n_draft, parent, n_live, cache: "Cache", O, ws, stream=None) -> None:
    e, B, d = _ELT.get(prm.dtype), prm.batch, prm.head_dim
    qs, ks, ps = (B, prm.n_q_heads, n_draft, d), (B, prm.n_kv_heads, n_draft, d), (B, n_draft)
    try:
        here = q.get_device()
        good = (here >= 0 and here == _current_device() and _ok(q, here, e, qs) and _ok(k_draft, here, e, ks)
                and _ok(v_draft, here, e, ks) and _ok(O, here, e, qs) and _ok(parent, here, _I32, ps)
                and (n_live is None or _ok(n_live, here, _I32, (B,))) and _ok(ws, here, _U8, ws.shape) and _fits(cache, here, e, d))
    except AttributeError:
        good = False
    if not good:
        _refuse_cache("tca_attn_tree", prm, cache, ("q", q, e, qs, True), ("k_draft", k_draft, e, ks, True), ("v_draft", v_draft, e, ks, True),
                ("O", O, e, qs, True), ("parent", parent, _I32, ps, True), ("n_live", n_live, _I32, (B,), True),
                ("ws", ws, _U8, None, True))
    _check(lib().tca_attn_tree(C.byref(prm), q.data_ptr(), k_draft.data_ptr(), v_draft.data_ptr(), n_draft, parent.data_ptr(),
                               None if n_live is None else n_live.data_ptr(), C.byref(cache.desc), O.data_ptr(),
                               ws.data_ptr(), ws.numel(), _stream_on(here, stream)), "tca_attn_tree")


def tca_cache_accept(prm, cache: "Cache", k_draft, v_draft, q_draft, n_draft, path, n_accept, stream=None) -> None:
    """path a CUDA int32 tensor [batch, n_draft]; n_accept an int32 numpy array of prm.batch elements."""
    e, B, d = _ELT.get(prm.dtype), prm.batch, prm.head_dim
    qs, ks, ps = (B, prm.n_q_heads, n_draft, d), (B, prm.n_kv_heads, n_draft, d), (B, n_draft)
    try:
        here = k_draft.get_device()
        good = (here >= 0 and here == _current_device() and _ok(k_draft, here, e, ks) and _ok(v_draft, here, e, ks)
                and _ok(q_draft, here, e, qs) and _ok(path, here, _I32, ps) and _fits(cache, here, e, d))
    except AttributeError:
        good = False
    if not good:
        _refuse_cache("tca_cache_accept", prm, cache, ("k_draft", k_draft, e, ks, True), ("v_draft", v_draft, e, ks, True),
                ("q_draft", q_draft, e, qs, True), ("path", path, _I32, ps, True))
    counts = _host_in("tca_cache_accept", "n_accept", n_accept, np.int32, B)
    _check(lib().tca_cache_accept(C.byref(prm), C.byref(cache.desc), k_draft.data_ptr(), v_draft.data_ptr(),
                                  q_draft.data_ptr(), n_draft, path.data_ptr(), counts, _stream_on(here, stream)),
           "tca_cache_accept")


def _refuse_paged(where: str, prm, cache: "PagedCache", *specs) -> None:
    e, here = _ELT.get(prm.dtype), torch.cuda.current_device() if torch.cuda.is_available() else -2
    if not isinstance(cache, PagedCache) or not cache.fits(here, e, prm.head_dim):
        raise ValueError(f"{where}: the cache must be a PagedCache on the current CUDA device, made for {e} and head size {prm.head_dim}")
    _refuse(where, *specs)


def tca_paged_append(prm, K, V, rows, seq_start, slots, mass, cache: "PagedCache", stream=None) -> None:
    """K, V [n_kv_heads, rows, d] as in tca_attn_packed; seq_start an int64 numpy array, or None: one row for each of
    `rows` sequences; slots an int32 numpy array or None; mass a float32 CUDA tensor [n_kv_heads, rows] or None."""
    e, ks, ms = _ELT.get(prm.dtype), (prm.n_kv_heads, rows, prm.head_dim), (prm.n_kv_heads, rows)
    try:
        here = K.get_device()
        good = (here >= 0 and here == _current_device() and (sk := _strides(K, here, e, ks)) and (sv := _strides(V, here, e, ks))
                and (mass is None or _ok(mass, here, _F32, ms)) and cache.fits(here, e, prm.head_dim))
    except AttributeError:
        good = False
    if not good:
        _refuse_paged("tca_paged_append", prm, cache, ("K", K, e, ks, False), ("V", V, e, ks, False), ("mass", mass, _F32, ms, True))
    if seq_start is None:
        n_seq, starts = rows, None
    else:
        n_seq = len(seq_start) - 1 if isinstance(seq_start, np.ndarray) and seq_start.ndim == 1 else -1
        starts = _host_in("tca_paged_append", "seq_start", seq_start, np.int64, n_seq + 1)
    places = None if slots is None else _host_in("tca_paged_append", "slots", slots, np.int32, n_seq)
    _check(lib().tca_paged_append(C.byref(prm), K.data_ptr(), V.data_ptr(), rows, _pack4(*sk, *sv), starts, places, n_seq,
                                  None if mass is None else mass.data_ptr(), C.byref(cache.desc), _stream_on(here, stream)),
           "tca_paged_append")


def tca_attn_paged_workspace_bytes(prm, cache: "PagedCache", accumulate) -> int:
    return int(lib().tca_attn_paged_workspace_bytes(C.byref(prm), C.byref(cache.desc), int(bool(accumulate))))


def alloc_paged_workspace(prm: tca_params, cache: "PagedCache", accumulate: bool = False) -> torch.Tensor:
    """A zero-filled workspace for tca_attn_paged calls over this cache (with accumulate, for calls of both kinds), or
    over any that need no more."""
    n = tca_attn_paged_workspace_bytes(prm, cache, accumulate)
    if n == 0:
        raise TcaError(TCA_ERR_INVALID_ARG, "tca_attn_paged_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=cache.k.device)


def tca_attn_paged(prm, q, cache: "PagedCache", n_sink, accumulate, O, ws, stream=None) -> None:
    """q, O [batch, n_q_heads, d], contiguous.  prm.window goes by slots: over a cache that is evicted from it is 2^31 - 1."""
    e, qs = _ELT.get(prm.dtype), (prm.batch, prm.n_q_heads, prm.head_dim)
    try:
        here = q.get_device()
        good = (here >= 0 and here == _current_device() and _ok(q, here, e, qs) and _ok(O, here, e, qs) and _ok(ws, here, _U8, ws.shape)
                and cache.fits(here, e, prm.head_dim))
    except AttributeError:
        good = False
    if not good:
        _refuse_paged("tca_attn_paged", prm, cache, ("q", q, e, qs, True), ("O", O, e, qs, True), ("ws", ws, _U8, None, True))
    _check(lib().tca_attn_paged(C.byref(prm), q.data_ptr(), C.byref(cache.desc), n_sink, 1 if accumulate else 0, O.data_ptr(),
                                ws.data_ptr(), ws.numel(), _stream_on(here, stream)), "tca_attn_paged")


def tca_paged_evict(prm, cache: "PagedCache", n_sink, n_recent, budget, stream=None) -> None:
    """budget an int32 CUDA tensor of one element per (sequence, KV head)."""
    e, bs = _ELT.get(prm.dtype), (prm.batch * prm.n_kv_heads,)
    try:
        here = budget.get_device()
        good = here >= 0 and here == _current_device() and _ok(budget, here, _I32, bs) and cache.fits(here, e, prm.head_dim)
    except AttributeError:
        good = False
    if not good:
        _refuse_paged("tca_paged_evict", prm, cache, ("budget", budget, _I32, bs, True))
    _check(lib().tca_paged_evict(C.byref(prm), C.byref(cache.desc), n_sink, n_recent, budget.data_ptr(), _stream_on(here, stream)),
           "tca_paged_evict")


def tca_paged_status(cache: "PagedCache", stream=None):
    """(status, detail) with detail = [unit, which check] when status is TCA_ERR_BOUNDS."""
    detail = np.zeros(2, dtype=np.int64)
    st = lib().tca_paged_status(C.byref(cache.desc), _stream(stream), detail.ctypes.data)
    return st, detail


# ----------------------------------------------------------------------------- cache descriptor holder
class Cache:
    """Owns the buffers a ``tca_cache_desc`` points at (torch device tensors, numpy host
    arrays) and keeps them alive.  Layout per unit: ``global_cap[u]`` rows for the global
    subset followed by ``tail_cap`` ring rows; segments are laid out back to back."""

    def __init__(self, prm: tca_params, global_cap: Sequence[int], tail_cap: int, t_keep: Sequence[int],
                 device="cuda", init: bool = True):
        U = prm.batch * prm.n_kv_heads
        gcap = np.ascontiguousarray(global_cap, dtype=np.int64)
        if gcap.shape != (U,):
            raise ValueError("global_cap must have one entry per (sequence, KV head)")
        self.prm = prm
        self.global_cap = gcap
        self.tail_cap = int(tail_cap)
        seg = np.zeros(U, dtype=np.int64)
        seg[1:] = np.cumsum(gcap[:-1] + self.tail_cap)
        self.seg_start = seg
        self.rows_total = int(seg[-1] + gcap[-1] + self.tail_cap)
        self.n_global = np.zeros(U, dtype=np.int64)
        self.tail_head = np.zeros(U, dtype=np.int64)
        self.n_tail = np.zeros(U, dtype=np.int64)
        self.seq_len = np.zeros(U, dtype=np.int64)
        self.t_keep = np.ascontiguousarray(t_keep, dtype=np.int64)
        tdt = torch.bfloat16 if prm.dtype == TCA_BF16 else torch.float32
        self.k = torch.zeros(self.rows_total, prm.head_dim, dtype=tdt, device=device)
        self.v = torch.zeros(self.rows_total, prm.head_dim, dtype=tdt, device=device)
        self.pos = torch.full((self.rows_total,), -1, dtype=torch.int32, device=device)
        self.state = torch.zeros(U * TCA_STATE_WORDS, dtype=torch.int64, device=device)
        self.desc = tca_cache_desc(
            self.k.data_ptr(), self.v.data_ptr(), self.pos.data_ptr(), self.state.data_ptr(),
            self.rows_total, U, self.tail_cap, self.seg_start.ctypes.data, self.global_cap.ctypes.data,
            self.n_global.ctypes.data, self.tail_head.ctypes.data, self.n_tail.ctypes.data,
            self.seq_len.ctypes.data, self.t_keep.ctypes.data)
        if init:
            tca_cache_init(prm, self)

    def unit_rows(self, u: int) -> np.ndarray:
        """Physical cache rows of unit u in logical order (global rows, then tail oldest first)."""
        g = self.seg_start[u] + np.arange(self.n_global[u])
        ring = self.seg_start[u] + self.global_cap[u]
        t = ring + (self.tail_head[u] + np.arange(self.n_tail[u])) % self.tail_cap
        return np.concatenate([g, t]).astype(np.int64)


class PagedCache:
    """Owns the buffers a ``tca_paged_desc`` points at and deals the pages of the pool to units.

    ``table``, ``state`` (rows, next position, first failed check, a word of the library's), ``pos`` and ``mass`` are
    device tensors; the last three lie in one buffer, ``meta``.  ``reserve`` and ``release`` keep a host copy of the table and a
    list of free pages, and upload the units that changed; a program with an allocator of its own writes ``table``
    instead.  They upload on ``stream``, or on torch's current one, and give pages to other units at once, so that
    stream has to be the calls' over the cache, or ordered with it."""

    def __init__(self, prm: tca_params, n_pages: int, page_size: int, max_pages: int, device="cuda"):
        U = prm.batch * prm.n_kv_heads
        n_pages, page_size, max_pages = int(n_pages), int(page_size), int(max_pages)
        if n_pages < 1 or page_size < 1 or max_pages < 1:
            raise ValueError("n_pages, page_size and max_pages must be positive")
        self.prm, self.n_pages, self.page_size, self.max_pages = prm, n_pages, page_size, max_pages
        tdt, n = _ELT[prm.dtype], n_pages * page_size
        self.k = torch.zeros(n_pages, page_size, prm.head_dim, dtype=tdt, device=device)
        self.v = torch.zeros(n_pages, page_size, prm.head_dim, dtype=tdt, device=device)
        pad = -n % 4                                     # the state begins on 16 bytes
        self.meta = torch.zeros(2 * (n + pad) + TCA_PG_STATE_WORDS * U, dtype=torch.int32, device=device)
        self.pos = self.meta[:n].view(n_pages, page_size)
        self.mass = self.meta[n + pad:2 * n + pad].view(torch.float32).view(n_pages, page_size)
        self.state = self.meta[2 * (n + pad):].view(U, TCA_PG_STATE_WORDS)
        self.table = torch.full((U, max_pages), -1, dtype=torch.int32, device=device)
        self.table_host = np.full((U, max_pages), -1, dtype=np.int32)
        self.n_held = np.zeros(U, dtype=np.int64)        # pages dealt to each unit
        self.free = list(range(n_pages - 1, -1, -1))
        self.desc = tca_paged_desc(self.k.data_ptr(), self.v.data_ptr(), self.pos.data_ptr(), self.mass.data_ptr(),
                                   self.table.data_ptr(), self.state.data_ptr(), n_pages, U, page_size, max_pages)
        self._kind = (self.k.get_device(), tdt, prm.head_dim)

    def fits(self, here, dtype, d) -> bool:
        """It lies on device `here` and was made for this type and head size."""
        return self._kind == (here, dtype, d)

    def reserve(self, rows: Sequence[int], stream=None) -> None:
        """Every unit u gets the pages that rows[u] rows need, where it has fewer."""
        want = self._pages(rows)
        more = np.maximum(0, want - self.n_held)
        if want.max(initial=0) > self.max_pages or more.sum() > len(self.free):
            raise TcaError(TCA_ERR_CAPACITY, "PagedCache.reserve")
        changed = np.nonzero(more)[0]
        for u in changed:
            n = int(more[u])
            self.table_host[u, self.n_held[u]:want[u]] = self.free[-n:][::-1]
            del self.free[-n:]
            self.n_held[u] = want[u]
        self._upload(changed, stream)

    def release(self, rows: Sequence[int], stream=None) -> None:
        """Every unit u gives back the pages that rows[u] rows do not need (after an eviction to a budget, or with 0
        rows when its sequence ends; its state is the caller's to clear then)."""
        want = self._pages(rows)
        changed = np.nonzero(want < self.n_held)[0]
        for u in changed:
            self.free.extend(self.table_host[u, want[u]:self.n_held[u]][::-1].tolist())
            self.table_host[u, want[u]:] = -1
            self.n_held[u] = want[u]
        self._upload(changed, stream)

    def _pages(self, rows) -> np.ndarray:
        rows = np.asarray(rows, dtype=np.int64)
        if rows.shape != self.n_held.shape or rows.min(initial=0) < 0:
            raise ValueError("rows must have one entry, not negative, per (sequence, KV head)")
        return -(-rows // self.page_size)

    def _upload(self, units, stream) -> None:
        if len(units):
            with torch.cuda.stream(stream):              # None: the current one
                at = torch.from_numpy(np.ascontiguousarray(units)).to(self.table.device)
                self.table[at] = torch.from_numpy(self.table_host[units]).to(self.table.device)


def tca_calib_colmean(prm, Q, K, L, colmean, ws, stream=None) -> None:
    _check(lib().tca_calib_colmean(C.byref(prm), _dev(Q), _dev(K), L, _dev(colmean), *_ws_args(ws), _stream(stream)),
           "tca_calib_colmean")


def tca_calib_score(prm, colmean, L, idx, offsets_dev, a_out, stream=None) -> None:
    _check(lib().tca_calib_score(C.byref(prm), _dev(colmean), L, _dev(idx), _dev(offsets_dev), _dev(a_out),
                                 _stream(stream)), "tca_calib_score")


def tca_calib_choose(a: np.ndarray, sizes: np.ndarray, tau: float) -> int:
    a = np.ascontiguousarray(a, dtype=np.float64)
    sizes = np.ascontiguousarray(sizes, dtype=np.int64)
    r = lib().tca_calib_choose(a.ctypes.data, sizes.ctypes.data, len(a), float(tau))
    if r < 0:
        raise TcaError(r, "tca_calib_choose")
    return int(r)


def tca_calib_candidates(block: int, n_candidates: int = 14, sigma: float = 1.0) -> np.ndarray:
    nK = int(block).bit_length()
    p = np.zeros((n_candidates, nK), dtype=np.float64)
    _check(lib().tca_calib_candidates(block, n_candidates, float(sigma), p.ctypes.data), "tca_calib_candidates")
    return p
