"""Python binding of libopattr, the GPU trace join for hardware-attributed
operator profiling ("Hardware-Attributed Operator Profiling for PyTorch").

Argument marshalling only: every step of the join runs in the CUDA kernels of
``libopattr.so`` (``csrc/``), reached through its C ABI (``include/opattr.h``).
PyTorch supplies device memory and the stream.  There is no CPU fallback: if
the library cannot be loaded the import of the binding's functions raises.

Function names follow the C ABI: ``opattr_create``, ``opattr_enclose``,
``opattr_match``, ``opattr_aggregate``, ``opattr_destroy``; ``Context`` wraps
them for torch tensors.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from dataclasses import dataclass

from . import _build

__all__ = [
    "OK", "W_COUNT_MISMATCH", "W_DEDUP_MISMATCH", "E_INVALID_ARG", "E_NOT_NESTED", "E_DEPTH",
    "E_COUNT_MISMATCH", "E_CUDA", "E_OOM", "E_TIMEOUT", "E_STATE", "E_PAGES", "OP_STRUCTURAL", "OP_NONOP",
    "N_COUNTERS", "OpattrError", "Context", "KVCache", "library", "build",
    "opattr_create", "opattr_enclose", "opattr_match", "opattr_aggregate", "opattr_join", "opattr_destroy",
    "opattr_status_string", "opattr_match_noalloc", "MATCH_NOALLOC_MAX", "opattr_attention", "opattr_cache_attention",
    "opattr_cache_append", "opattr_cache_fork", "opattr_cache_trim", "opattr_cache_compact", "opattr_check",
]

OK, W_COUNT_MISMATCH, W_DEDUP_MISMATCH = 0, 1, 2
E_INVALID_ARG, E_NOT_NESTED, E_DEPTH, E_COUNT_MISMATCH = -1, -2, -3, -4
E_CUDA, E_OOM, E_TIMEOUT, E_STATE, E_PAGES = -5, -6, -7, -8, -9
OP_STRUCTURAL = 0xFFFFFFFF
OP_NONOP = 0xFFFFFFFE
N_COUNTERS = 20
OP_NONE = 0xFFFFFFFF
TIER_NONE, TIER_HIGH, TIER_NVTX, TIER_INDUCTOR = 0, 1, 2, 3
MATCH_NOALLOC_MAX = 65536
MISMATCH = {"skip_name": 0, "prefix": 1, "error": 2}

_vp = ctypes.c_void_p


class Kernels(ctypes.Structure):
    _fields_ = [("stream", _vp), ("start_ns", _vp), ("dur_ns", _vp), ("name_id", _vp), ("layer_id", _vp),
                ("n", ctypes.c_int64)]


class Ranges(ctypes.Structure):
    _fields_ = [("stream", _vp), ("start_ns", _vp), ("end_ns", _vp), ("depth", _vp), ("op_id", _vp),
                ("n", ctypes.c_int64)]


class Ncu(ctypes.Structure):
    _fields_ = [("name_id", _vp), ("counters", _vp), ("n", ctypes.c_int64), ("stream", _vp)]


class Dedup(ctypes.Structure):
    _fields_ = [("class_of_layer", _vp), ("rep_of_class", _vp), ("n_layers", ctypes.c_int32),
                ("n_classes", ctypes.c_int32)]


class Config(ctypes.Structure):
    _fields_ = [("mismatch", ctypes.c_int), ("dedup", ctypes.c_int32), ("checked", ctypes.c_int32),
                ("spin_limit", ctypes.c_int64)]


class MatchSummary(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int64) for f in ("kernels", "replayed", "direct", "broadcast", "unmatched",
                                              "names_mismatched", "count_unmatched", "dedup_mismatch")] + \
               [("fast_path", ctypes.c_int32), ("reserved", ctypes.c_int32)]

    def as_dict(self) -> dict:
        return {"kernels": self.kernels, "replayed": self.replayed, "direct": self.direct, "broadcast": self.broadcast,
                "unmatched": self.unmatched, "names_mismatched": self.names_mismatched,
                "count_unmatched": self.count_unmatched, "dedup_mismatch": self.dedup_mismatch,
                "fast_path": self.fast_path}


class Corr(ctypes.Structure):
    _fields_ = [("name_id", _vp), ("invocation", _vp), ("op_id", _vp), ("n", ctypes.c_int64)]


class Fusion(ctypes.Structure):
    _fields_ = [("op_of_name", _vp), ("list_len", _vp), ("n_names", ctypes.c_int64)]


class AttrSummary(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int64) for f in ("kernels", "high", "nvtx", "inductor", "none", "fused", "corr_used")]

    def as_dict(self) -> dict:
        return {f: int(getattr(self, f)) for f, _ in self._fields_}


class ProfileMeta(ctypes.Structure):
    _fields_ = [("model_name", ctypes.c_char_p), ("device_name", ctypes.c_char_p), ("compile_mode", ctypes.c_char_p),
                ("capture_timestamp_utc", ctypes.c_char_p), ("include_kernels", ctypes.c_int32)]


class ProfileNames(ctypes.Structure):
    _fields_ = [("kernel_name", _vp), ("n_kernel_names", ctypes.c_int64), ("op_name", _vp),
                ("op_call_index", _vp)]


class OpAggregates(ctypes.Structure):
    _fields_ = [("kernel_count", _vp), ("total_duration_ns", _vp), ("matched_count", _vp), ("agg", _vp)]


class Totals(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int64) for f in ("total_ns", "attributed_ns", "unattributed_ns", "kernels",
                                              "attributed_kernels", "matched_kernels")] + \
               [("attributed_frac", ctypes.c_double), ("unattributed_frac", ctypes.c_double)]

    def as_dict(self) -> dict:
        return {"total_ns": self.total_ns, "attributed_ns": self.attributed_ns, "unattributed_ns": self.unattributed_ns,
                "kernels": self.kernels, "attributed_kernels": self.attributed_kernels,
                "matched_kernels": self.matched_kernels, "attributed_frac": self.attributed_frac,
                "unattributed_frac": self.unattributed_frac}


class Rows(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class Prompt(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("dtype", "n_seqs", "q_heads", "kv_heads", "head_dim", "causal")] + \
               [("scale", ctypes.c_float), ("reserved", ctypes.c_int32), ("q_tokens", ctypes.c_int64),
                ("k_tokens", ctypes.c_int64), ("q", Rows), ("k", Rows), ("v", Rows), ("out", Rows),
                ("q_offsets", _vp), ("k_offsets", _vp), ("lse", _vp)]


class Cache(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("dtype", "page_size", "kv_heads", "head_dim", "n_seqs",
                                              "pages_per_seq")] + \
               [("n_pages", ctypes.c_int64)] + \
               [(f, _vp) for f in ("k_pages", "v_pages", "table", "length", "refs", "low")]


_lib_lock = threading.Lock()
_lib = None


def build(force: bool = False) -> str:
    """Compile libopattr.so for sm_103a (no-op when up to date)."""
    return _build.build(force=force)


def library():
    """Load libopattr.so (building it first if needed).  Raises on failure."""
    global _lib
    with _lib_lock:
        if _lib is None:
            path = _build.LIB
            if not os.path.exists(path) or os.environ.get("OPATTR_REBUILD"):
                path = _build.build()
            lib = ctypes.CDLL(path)
            P = ctypes.POINTER
            lib.opattr_create.argtypes = [P(_vp), ctypes.c_int, _vp, P(Config)]
            lib.opattr_enclose.argtypes = [_vp, P(Kernels), P(Ranges), _vp, _vp]
            lib.opattr_match.argtypes = [_vp, P(Kernels), P(Ncu), P(Dedup), _vp, _vp, P(MatchSummary)]
            lib.opattr_aggregate.argtypes = [_vp, P(Kernels), P(Ranges), _vp, P(Ncu), _vp, ctypes.c_uint32,
                                             P(OpAggregates), P(Totals)]
            lib.opattr_join.argtypes = [_vp, P(Kernels), P(Ranges), P(Ncu), P(Dedup), ctypes.c_uint32, _vp, _vp, _vp,
                                        _vp, P(OpAggregates), P(MatchSummary), P(Totals)]
            lib.opattr_attribute.argtypes = [_vp, P(Kernels), P(Ranges), _vp, _vp, P(Corr), P(Fusion),
                                             ctypes.c_uint32, _vp, _vp, _vp, _vp, P(AttrSummary)]
            lib.opattr_rollup.argtypes = [_vp, P(Kernels), P(Ranges), _vp, P(Ncu), _vp, ctypes.c_uint32, _vp,
                                          ctypes.c_uint32, P(OpAggregates)]
            lib.opattr_write_profile.argtypes = [ctypes.c_char_p, P(ProfileMeta), P(ProfileNames), P(Kernels), _vp,
                                                 _vp, _vp, _vp, _vp, _vp, ctypes.c_int64, ctypes.c_uint32,
                                                 P(OpAggregates), P(ctypes.c_int64)]
            lib.opattr_write_profile.restype = ctypes.c_int
            lib.opattr_destroy.argtypes = [_vp]
            lib.opattr_destroy.restype = None
            lib.opattr_status_string.argtypes = [ctypes.c_int]
            lib.opattr_status_string.restype = ctypes.c_char_p
            lib.opattr_set_timing.argtypes = [_vp, ctypes.c_int]
            lib.opattr_set_timing_only.argtypes = [_vp, ctypes.c_char_p]
            lib.opattr_set_timing_only.restype = ctypes.c_int
            lib.opattr_timing_report.argtypes = [_vp, P(ctypes.c_char_p), P(ctypes.c_double), P(ctypes.c_int64),
                                                 ctypes.c_int]
            lib.opattr_timing_reset.argtypes = [_vp]
            lib.opattr_timing_reset.restype = None
            lib.opattr_launch_count.argtypes = [_vp]
            lib.opattr_launch_count.restype = ctypes.c_int64
            lib.opattr_match_noalloc.argtypes = [P(Kernels), P(Ncu), ctypes.c_int, _vp, _vp, P(MatchSummary), _vp]
            lib.opattr_match_noalloc.restype = ctypes.c_int
            i32, i64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
            # (structs of these calls go by reference, or packed into bytes)
            lib.opattr_attention.argtypes = [_vp, _vp]
            lib.opattr_cache_attention.argtypes = [_vp, _vp, _vp, i32, i32, _vp, _vp, _vp, f32]
            lib.opattr_cache_append.argtypes = [_vp, _vp, _vp, i32, _vp, i64, _vp, _vp]
            lib.opattr_cache_fork.argtypes = [_vp, _vp, _vp, _vp, i32]
            lib.opattr_cache_trim.argtypes = [_vp, _vp, _vp, _vp, i32]
            lib.opattr_cache_compact.argtypes = [_vp, _vp, _vp]
            lib.opattr_check.argtypes = [_vp]
            for f in ("opattr_create", "opattr_enclose", "opattr_match", "opattr_aggregate", "opattr_attribute",
                      "opattr_rollup", "opattr_set_timing", "opattr_timing_report", "opattr_attention",
                      "opattr_cache_attention", "opattr_cache_append", "opattr_cache_fork", "opattr_cache_trim",
                      "opattr_cache_compact", "opattr_check"):
                getattr(lib, f).restype = ctypes.c_int
            _lib = lib
        return _lib


class OpattrError(RuntimeError):
    def __init__(self, status: int, call: str):
        super().__init__(f"{call}: {opattr_status_string(status)} ({status})")
        self.status = status


def opattr_status_string(status: int) -> str:
    return library().opattr_status_string(status).decode()


# ---------------------------------------------------------------- C ABI, one to one
def opattr_create(device: int = 0, stream: int | None = None, mismatch: str = "skip_name", dedup: bool = True,
                  spin_limit: int = 0):
    """Returns (status, handle)."""
    cfg = Config(MISMATCH[mismatch], int(bool(dedup)), 0, int(spin_limit))
    h = _vp()
    st = library().opattr_create(ctypes.byref(h), int(device), _vp(stream or 0), ctypes.byref(cfg))
    return st, h


def opattr_enclose(handle, kernels: Kernels, ranges: Ranges, range_of_kernel_ptr: int, n_op_ptr: int | None) -> int:
    return (_lib or library()).opattr_enclose(handle, ctypes.byref(kernels), ctypes.byref(ranges), range_of_kernel_ptr,
                                              n_op_ptr)


def opattr_match(handle, kernels: Kernels, ncu: Ncu, dedup: Dedup | None, idx_ptr: int, kind_ptr: int | None,
                 summary: MatchSummary) -> int:
    return (_lib or library()).opattr_match(handle, ctypes.byref(kernels), ctypes.byref(ncu),
                                            ctypes.byref(dedup) if dedup is not None else None, idx_ptr,
                                            kind_ptr, ctypes.byref(summary))


def opattr_aggregate(handle, kernels: Kernels, ranges: Ranges, rok_ptr: int, ncu: Ncu, idx_ptr: int, n_ops: int,
                     out: OpAggregates, totals: Totals) -> int:
    return (_lib or library()).opattr_aggregate(handle, ctypes.byref(kernels), ctypes.byref(ranges), rok_ptr,
                                                ctypes.byref(ncu), idx_ptr, ctypes.c_uint32(n_ops), ctypes.byref(out),
                                                ctypes.byref(totals))


def opattr_join(handle, kernels: Kernels, ranges: Ranges, ncu: Ncu, dedup: Dedup | None, n_ops: int, rok_ptr: int,
                nop_ptr: int | None, idx_ptr: int, kind_ptr: int | None, out: OpAggregates, summary: MatchSummary,
                totals: Totals) -> int:
    return (_lib or library()).opattr_join(handle, ctypes.byref(kernels), ctypes.byref(ranges), ctypes.byref(ncu),
                                           ctypes.byref(dedup) if dedup is not None else None, ctypes.c_uint32(n_ops),
                                           rok_ptr, nop_ptr, idx_ptr, kind_ptr, ctypes.byref(out),
                                           ctypes.byref(summary), ctypes.byref(totals))


def opattr_attribute(handle, kernels: Kernels, ranges: Ranges, rok_ptr: int, nop_ptr: int | None,
                     corr: Corr | None, fusion: Fusion | None, n_ops: int, op_ptr: int, tier_ptr: int | None,
                     fused_with_ptr: int | None, is_fused_ptr: int | None, summary: AttrSummary) -> int:
    return (_lib or library()).opattr_attribute(handle, ctypes.byref(kernels), ctypes.byref(ranges), rok_ptr,
                                                nop_ptr, ctypes.byref(corr) if corr is not None else None,
                                                ctypes.byref(fusion) if fusion is not None else None,
                                                ctypes.c_uint32(n_ops), op_ptr, tier_ptr, fused_with_ptr, is_fused_ptr,
                                                ctypes.byref(summary))


def opattr_rollup(handle, kernels: Kernels, ranges: Ranges, rok_ptr: int | None, ncu: Ncu, idx_ptr: int, n_ops: int,
                  class_ptr: int, n_classes: int, out: OpAggregates) -> int:
    return (_lib or library()).opattr_rollup(handle, ctypes.byref(kernels), ctypes.byref(ranges), rok_ptr,
                                             ctypes.byref(ncu), idx_ptr, ctypes.c_uint32(n_ops), class_ptr,
                                             ctypes.c_uint32(n_classes), ctypes.byref(out))


def write_profile(path: str, k_stream, k_dur, k_name, op_of_kernel, ncu_idx, counters, ops: dict, tier=None,
                  is_fused=None, fused_with=None, kernel_names=None, op_names=None, op_call_index=None,
                  meta: dict | None = None, include_kernels: bool = True) -> int:
    """profile.json (App. A.4) from HOST (numpy) arrays: opattr_write_profile.
    Returns the number of bytes written; raises OpattrError on failure."""
    import numpy as np
    c = lambda a, dt: None if a is None else np.ascontiguousarray(a).view(dt) if np.asarray(a).dtype.itemsize == \
        np.dtype(dt).itemsize else np.ascontiguousarray(a, dtype=dt)
    ks, kd, kn = c(k_stream, np.uint8), c(k_dur, np.int64), c(k_name, np.uint32)
    op, ni = c(op_of_kernel, np.uint32), c(ncu_idx, np.int32)
    cn = np.ascontiguousarray(counters, dtype=np.float32)
    tr, fz, fw = c(tier, np.uint8), c(is_fused, np.uint8), c(fused_with, np.uint32)
    kc, td, mc = (np.ascontiguousarray(ops[k], dtype=np.int64) for k in ("kernel_count", "total_duration_ns",
                                                                         "matched_count"))
    agg = np.ascontiguousarray(ops["agg"], dtype=np.float64)
    p = lambda a: None if a is None else a.ctypes.data
    K = len(kd)
    kern = Kernels(p(ks), None, p(kd), p(kn), None, K)
    out = OpAggregates(p(kc), p(td), p(mc), p(agg))
    keep = []
    names = ProfileNames(None, 0, None, None)
    if kernel_names is not None:
        arr = (ctypes.c_char_p * len(kernel_names))(*[s.encode() for s in kernel_names])
        keep.append(arr)
        names.kernel_name, names.n_kernel_names = ctypes.cast(arr, _vp), len(kernel_names)
    if op_names is not None:
        arr = (ctypes.c_char_p * len(op_names))(*[s.encode() for s in op_names])
        keep.append(arr)
        names.op_name = ctypes.cast(arr, _vp)
    ci = c(op_call_index, np.int64)
    if ci is not None:
        names.op_call_index = p(ci)
    m = meta or {}
    pm = ProfileMeta(*[(m.get(k).encode() if m.get(k) is not None else None)
                       for k in ("model_name", "device_name", "compile_mode", "capture_timestamp_utc")],
                     int(bool(include_kernels)))
    nbytes = ctypes.c_int64(0)
    st = library().opattr_write_profile(str(path).encode(), ctypes.byref(pm), ctypes.byref(names), ctypes.byref(kern),
                                        p(op), p(tr), p(fz), p(fw), p(ni), p(cn), cn.shape[0] if cn.ndim == 2 else
                                        cn.size // N_COUNTERS, int(len(kc)), ctypes.byref(out), ctypes.byref(nbytes))
    del keep
    if st != OK:
        raise OpattrError(st, "opattr_write_profile")
    return int(nbytes.value)


def opattr_match_noalloc(kernels: Kernels, ncu: Ncu, mismatch: str, idx_ptr: int, kind_ptr: int | None,
                         summary: MatchSummary, stream: int | None) -> int:
    """opattr_match without a context and without any device allocation, for
    callers that must not allocate (see include/opattr.h); inputs of at most
    OPATTR_MATCH_NOALLOC_MAX kernels and rows."""
    return library().opattr_match_noalloc(ctypes.byref(kernels), ctypes.byref(ncu), MISMATCH[mismatch],
                                          _vp(idx_ptr), _vp(kind_ptr or 0), ctypes.byref(summary), _vp(stream or 0))


def opattr_attention(handle, args) -> int:
    """args: a Prompt (by reference) or its bytes."""
    return (_lib or library()).opattr_attention(handle, args)


def opattr_cache_attention(handle, cache, seqs_ptr: int | None, n: int, q_heads: int, q, out, lse_ptr: int | None,
                           scale: float) -> int:
    """cache: a Cache by reference; q, out: Rows by reference, or their bytes."""
    return (_lib or library()).opattr_cache_attention(handle, cache, seqs_ptr, n, q_heads, q, out, lse_ptr, scale)


def opattr_cache_append(handle, cache, seqs_ptr: int, n: int, offsets_ptr: int, tokens: int, k, v) -> int:
    return (_lib or library()).opattr_cache_append(handle, cache, seqs_ptr, n, offsets_ptr, tokens, k, v)


def opattr_cache_fork(handle, cache, src_ptr: int, dst_ptr: int, n: int) -> int:
    return (_lib or library()).opattr_cache_fork(handle, cache, src_ptr, dst_ptr, n)


def opattr_cache_trim(handle, cache, seqs_ptr: int, lengths_ptr: int | None, n: int) -> int:
    return (_lib or library()).opattr_cache_trim(handle, cache, seqs_ptr, lengths_ptr, n)


def opattr_cache_compact(handle, cache, live_ptr: int | None) -> int:
    return (_lib or library()).opattr_cache_compact(handle, cache, live_ptr)


def opattr_check(handle) -> int:
    return (_lib or library()).opattr_check(handle)


def opattr_destroy(handle) -> None:
    if handle:
        library().opattr_destroy(handle)


# ---------------------------------------------------------------- torch convenience layer
def _ptr(t, dtype, name, device):
    if t is None:
        return None
    if t.dtype is not dtype and not (dtype is _torch().uint32 and t.dtype is _torch().int32):
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.get_device() != device:                 # -1 for a host tensor
        raise ValueError(f"{name}: must live on cuda:{device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr() if t.numel() else None


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


@dataclass
class DeviceTrace:
    """A trace's arrays as device tensors (see include/opattr.h for layouts)."""
    k_stream: object
    k_start: object
    k_dur: object
    k_name: object
    k_layer: object
    r_stream: object
    r_start: object
    r_end: object
    r_depth: object
    r_op: object
    n_ops: int
    ncu_name: object
    counters: object
    class_of_layer: object = None   # host (numpy / list) tables
    rep_of_class: object = None
    ncu_stream: object = None       # stream of each ncu row (per-stream replay runs), or None
    corr_name: object = None        # torch.profiler correlation map (HIGH tier), or None
    corr_inv: object = None
    corr_op: object = None
    fusion_op: object = None        # Inductor fusion map per name id (INDUCTOR tier), or None
    fusion_len: object = None

    @property
    def K(self):
        return int(self.k_start.shape[0])

    @property
    def R(self):
        return int(self.r_start.shape[0])

    @property
    def M(self):
        return int(self.ncu_name.shape[0])


def to_device(trace, device: int = 0, pin: bool = False) -> DeviceTrace:
    """Copy a tracegen.Trace (numpy arrays) to the GPU as torch tensors."""
    import torch

    def d(a):
        if a is None:
            return None
        t = torch.from_numpy(a)
        if pin:
            t = t.pin_memory()
        return t.to(f"cuda:{device}", non_blocking=pin)

    return DeviceTrace(d(trace.k_stream), d(trace.k_start), d(trace.k_dur), d(trace.k_name), d(trace.k_layer),
                       d(trace.r_stream), d(trace.r_start), d(trace.r_end), d(trace.r_depth), d(trace.r_op),
                       int(trace.n_ops), d(trace.ncu_name), d(trace.counters), trace.class_of_layer,
                       trace.rep_of_class, d(getattr(trace, "ncu_stream", None)), d(getattr(trace, "corr_name", None)),
                       d(getattr(trace, "corr_inv", None)), d(getattr(trace, "corr_op", None)),
                       d(getattr(trace, "fusion_op", None)), d(getattr(trace, "fusion_len", None)))


def _dtype(t, name) -> int:
    """opattr_dtype of a tensor of 16-bit values."""
    torch = _torch()
    if t.dtype is torch.bfloat16:
        return 0
    if t.dtype is torch.float16:
        return 1
    raise TypeError(f"{name}: expected torch.bfloat16 or torch.float16, got {t.dtype}")


# Rows and Prompt as bytes: one call in the place of an object and its fields
_ROWS = struct.Struct("@Pqq")
_PROMPT = struct.Struct("@6ifi2q" + "Pqq" * 4 + "3P")


def _rows(t, heads: int | None, dim: int, like, name, device):
    """[tokens, heads, dim] of `like`'s type as the fields of opattr_rows; a view
    whose rows are contiguous and start 16 bytes apart or a multiple of that."""
    shape = t.shape
    if len(shape) != 3 or (heads is not None and shape[1] != heads) or shape[2] != dim:
        raise ValueError(f"{name}: expected [tokens, {heads if heads is not None else 'heads'}, {dim}], "
                         f"got {list(shape)}")
    if t.dtype is not like:
        raise TypeError(f"{name}: expected {like}, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name}: must live on cuda:{device}")
    st, sh, se = t.stride()
    n, h, _ = shape
    p = t.data_ptr()
    if n == 0 or h == 0:
        return 0, 0, 0
    if n == 1:
        st = h * dim
    if h == 1:
        sh = dim
    if se != 1 or p & 15 or st & 7 or sh & 7 or st < 8 or sh < 0:
        raise ValueError(f"{name}: a row's elements must be contiguous and rows 16-byte aligned")
    return p, st, sh


def _no_grad(**tensors):
    """These operators have no backward pass: where gradients are recorded, a
    result that is cut off from its inputs in silence would be wrong."""
    if _torch().is_grad_enabled():
        for name, t in tensors.items():
            if t.requires_grad:
                raise ValueError(f"{name}: requires a gradient, which this call has none of: use torch.no_grad() or detach it")


def _distinct(t, name):
    """An output's rows must not overlap."""
    if t.numel() and any(s == 0 and n > 1 for s, n in zip(t.stride(), t.shape)):
        raise ValueError(f"{name}: must not be expanded")


@dataclass
class KVCache:
    """A paged key-value cache as device tensors (opattr_cache in
    include/opattr.h has the layouts); Context.cache makes an empty one.  A field
    may be replaced by another tensor that fits the others."""
    k_pages: object                 # [n_pages, kv_heads, page_size, head_dim] bfloat16 or float16
    v_pages: object
    table: object                   # int32 [n_seqs, pages_per_seq], -1 past a sequence's length
    length: object                  # int32 [n_seqs]
    refs: object                    # int32 [n_pages]: sequences that hold a page
    low: object                     # int32 [1]: no page below it is free

    def __post_init__(self):
        self._lay_out()

    def __setattr__(self, name, value):
        old = self.__dict__.get(name)
        object.__setattr__(self, name, value)
        if "struct" in self.__dict__ and name in self.__dataclass_fields__ and value is not old:
            # the calls go by the struct's addresses
            try:
                self._lay_out()
            except Exception:
                object.__setattr__(self, name, old)
                raise

    def _lay_out(self):
        """Checks the tensors; their sizes and addresses as the calls take them."""
        dv = self.k_pages.get_device()
        if self.k_pages.dim() != 4 or self.v_pages.shape != self.k_pages.shape:
            raise ValueError("k_pages, v_pages: expected one shape [n_pages, kv_heads, page_size, head_dim]")
        dtype = _dtype(self.k_pages, "k_pages")
        n, g, page, dim = self.k_pages.shape
        torch = _torch()
        if page < 16 or page > 1024 or page & (page - 1):
            raise ValueError(f"page_size: expected a power of two from 16 to 1024, got {page}")
        if dim < 8 or dim > 128 or dim % 8:
            raise ValueError(f"head_dim: expected a multiple of 8 from 8 to 128, got {dim}")
        if self.table.dim() != 2 or self.length.shape != (self.table.shape[0],) or self.refs.shape != (n,) or \
                self.low.numel() != 1 or n < 1 or g < 1 or self.table.numel() < 1:
            raise ValueError("expected table [n_seqs, pages_per_seq], length [n_seqs], refs [n_pages], low [1]")
        self.struct = Cache(dtype, page, g, dim, self.table.shape[0], self.table.shape[1], n,
                            _ptr(self.k_pages, self.k_pages.dtype, "k_pages", dv),
                            _ptr(self.v_pages, self.k_pages.dtype, "v_pages", dv),
                            _ptr(self.table, torch.int32, "table", dv), _ptr(self.length, torch.int32, "length", dv),
                            _ptr(self.refs, torch.int32, "refs", dv), _ptr(self.low, torch.int32, "low", dv))
        self.device, self.by_ref = dv, ctypes.byref(self.struct)


class Context:
    """An opattr context bound to one device and one CUDA stream."""

    def __init__(self, device: int = 0, stream=None, mismatch: str = "skip_name", dedup: bool = True,
                 spin_limit: int = 0):
        import torch
        self.device = device
        self._dev = torch.device("cuda", device)
        if stream is None:
            stream = torch.cuda.current_stream(device)
        self.stream = stream
        self._raw_stream = stream.cuda_stream
        st, self.handle = opattr_create(device, stream.cuda_stream, mismatch, dedup, spin_limit)
        if st != OK:
            raise OpattrError(st, "opattr_create")

    def close(self):
        if getattr(self, "handle", None):
            opattr_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- structs
    def kernels(self, tr: DeviceTrace) -> Kernels:
        torch = _torch()
        dv = self.device
        return Kernels(_ptr(tr.k_stream, torch.uint8, "k_stream", dv), _ptr(tr.k_start, torch.int64, "k_start", dv),
                       _ptr(tr.k_dur, torch.int64, "k_dur", dv), _ptr(tr.k_name, torch.uint32, "k_name", dv),
                       _ptr(tr.k_layer, torch.int32, "k_layer", dv), tr.K)

    def ranges(self, tr: DeviceTrace) -> Ranges:
        torch = _torch()
        dv = self.device
        return Ranges(_ptr(tr.r_stream, torch.uint8, "r_stream", dv), _ptr(tr.r_start, torch.int64, "r_start", dv),
                      _ptr(tr.r_end, torch.int64, "r_end", dv), _ptr(tr.r_depth, torch.uint8, "r_depth", dv),
                      _ptr(tr.r_op, torch.uint32, "r_op", dv), tr.R)

    def ncu(self, tr: DeviceTrace) -> Ncu:
        torch = _torch()
        dv = self.device
        return Ncu(_ptr(tr.ncu_name, torch.uint32, "ncu_name", dv), _ptr(tr.counters, torch.float32, "counters", dv),
                   tr.M, _ptr(tr.ncu_stream, torch.uint8, "ncu_stream", dv))

    # -- calls
    def enclose(self, tr: DeviceTrace, out_range=None, out_nop=None, need_nop: bool = True):
        torch = _torch()
        dev = self._dev
        if out_range is None:
            out_range = torch.empty(tr.K, dtype=torch.int32, device=dev)
        if out_nop is None and need_nop:
            out_nop = torch.empty(tr.K, dtype=torch.uint8, device=dev)
        st = opattr_enclose(self.handle, self.kernels(tr), self.ranges(tr),
                            _ptr(out_range, torch.int32, "range_of_kernel", self.device),
                            _ptr(out_nop, torch.uint8, "n_op_enclosing", self.device) if out_nop is not None else None)
        if st < 0:
            raise OpattrError(st, "opattr_enclose")
        return st, out_range, out_nop

    @staticmethod
    def _dedup(tr: DeviceTrace, dedup: bool | None):
        """(Dedup struct or None, the host arrays it points into)."""
        import numpy as np
        use = (tr.class_of_layer is not None and tr.k_layer is not None) if dedup is None else dedup
        if not use:
            return None, None
        col = np.ascontiguousarray(tr.class_of_layer, dtype=np.int32)
        roc = np.ascontiguousarray(tr.rep_of_class, dtype=np.int32)
        return Dedup(col.ctypes.data if col.size else None, roc.ctypes.data if roc.size else None, len(col),
                     len(roc)), (col, roc)

    def match(self, tr: DeviceTrace, dedup: bool | None = None, out_idx=None, out_kind=None):
        torch = _torch()
        dev = self._dev
        if out_idx is None:
            out_idx = torch.empty(tr.K, dtype=torch.int32, device=dev)
        if out_kind is None:
            out_kind = torch.empty(tr.K, dtype=torch.uint8, device=dev)
        dd, keep = self._dedup(tr, dedup)
        summ = MatchSummary()
        st = opattr_match(self.handle, self.kernels(tr), self.ncu(tr), dd,
                          _ptr(out_idx, torch.int32, "ncu_idx_of_kernel", self.device),
                          _ptr(out_kind, torch.uint8, "match_kind", self.device), summ)
        del keep
        if st < 0:
            raise OpattrError(st, "opattr_match")
        return st, out_idx, out_kind, summ.as_dict()

    def join(self, tr: DeviceTrace, dedup: bool | None = None, out=None, ops=None):
        """enclose + match + aggregate in one call (opattr_join).  `out` may hold
        preallocated range_of_kernel / n_op_enclosing / ncu_idx / match_kind
        tensors; returns (status, out, ops, match summary, totals)."""
        torch = _torch()
        dev = self._dev
        dv = self.device
        out = dict(out or {})
        for k, dt in (("range_of_kernel", torch.int32), ("n_op_enclosing", torch.uint8), ("ncu_idx", torch.int32),
                      ("match_kind", torch.uint8)):
            if out.get(k) is None:
                out[k] = torch.empty(tr.K, dtype=dt, device=dev)
        if ops is None:
            ops = self.alloc_ops(tr.n_ops)
        agg = OpAggregates(_ptr(ops["kernel_count"], torch.int64, "kernel_count", dv),
                           _ptr(ops["total_duration_ns"], torch.int64, "total_duration_ns", dv),
                           _ptr(ops["matched_count"], torch.int64, "matched_count", dv),
                           _ptr(ops["agg"], torch.float64, "agg", dv))
        dd, keep = self._dedup(tr, dedup)
        summ, tot = MatchSummary(), Totals()
        st = opattr_join(self.handle, self.kernels(tr), self.ranges(tr), self.ncu(tr), dd, tr.n_ops,
                         _ptr(out["range_of_kernel"], torch.int32, "range_of_kernel", dv),
                         _ptr(out["n_op_enclosing"], torch.uint8, "n_op_enclosing", dv),
                         _ptr(out["ncu_idx"], torch.int32, "ncu_idx_of_kernel", dv),
                         _ptr(out["match_kind"], torch.uint8, "match_kind", dv), agg, summ, tot)
        del keep
        if st < 0:
            raise OpattrError(st, "opattr_join")
        return st, out, ops, summ.as_dict(), tot.as_dict()

    def alloc_ops(self, n_ops: int):
        torch = _torch()
        dev = self._dev
        return dict(kernel_count=torch.empty(n_ops, dtype=torch.int64, device=dev),
                    total_duration_ns=torch.empty(n_ops, dtype=torch.int64, device=dev),
                    matched_count=torch.empty(n_ops, dtype=torch.int64, device=dev),
                    agg=torch.empty((N_COUNTERS, n_ops), dtype=torch.float64, device=dev))

    def attribute(self, tr: DeviceTrace, range_of_kernel, n_op_enclosing=None, use_corr: bool = True,
                  use_fusion: bool = True, out=None):
        """The attribution tiers of Fig. 2: returns (status, op_of_kernel, tier, fused_with, is_fused, summary)."""
        torch = _torch()
        dv = self.device
        dev = self._dev
        if out is None:
            out = dict(op=torch.empty(tr.K, dtype=torch.int32, device=dev),
                       tier=torch.empty(tr.K, dtype=torch.uint8, device=dev),
                       fused_with=torch.empty(tr.K, dtype=torch.int32, device=dev),
                       is_fused=torch.empty(tr.K, dtype=torch.uint8, device=dev))
        corr = fusion = None
        if use_corr and tr.corr_name is not None:
            corr = Corr(_ptr(tr.corr_name, torch.uint32, "corr_name", dv), _ptr(tr.corr_inv, torch.uint32, "corr_inv", dv),
                        _ptr(tr.corr_op, torch.uint32, "corr_op", dv), int(tr.corr_name.shape[0]))
        if use_fusion and tr.fusion_op is not None:
            fusion = Fusion(_ptr(tr.fusion_op, torch.uint32, "fusion_op", dv),
                            _ptr(tr.fusion_len, torch.uint8, "fusion_len", dv), int(tr.fusion_op.shape[0]))
        summ = AttrSummary()
        st = opattr_attribute(self.handle, self.kernels(tr), self.ranges(tr),
                              _ptr(range_of_kernel, torch.int32, "range_of_kernel", dv),
                              _ptr(n_op_enclosing, torch.uint8, "n_op_enclosing", dv) if n_op_enclosing is not None
                              else None, corr, fusion, tr.n_ops, _ptr(out["op"], torch.uint32, "op_of_kernel", dv),
                              _ptr(out["tier"], torch.uint8, "tier", dv),
                              _ptr(out["fused_with"], torch.uint32, "fused_with", dv),
                              _ptr(out["is_fused"], torch.uint8, "is_fused", dv), summ)
        if st < 0:
            raise OpattrError(st, "opattr_attribute")
        return st, out["op"], out["tier"], out["fused_with"], out["is_fused"], summ.as_dict()

    def aggregate(self, tr: DeviceTrace, range_of_kernel, ncu_idx, ops=None, op_of_kernel=None):
        """Eq. (1) per operator.  With op_of_kernel (opattr_attribute's output)
        in place of range_of_kernel, each kernel's operator is taken from it."""
        torch = _torch()
        if ops is None:
            ops = self.alloc_ops(tr.n_ops)
        dv = self.device
        out = OpAggregates(_ptr(ops["kernel_count"], torch.int64, "kernel_count", dv),
                           _ptr(ops["total_duration_ns"], torch.int64, "total_duration_ns", dv),
                           _ptr(ops["matched_count"], torch.int64, "matched_count", dv),
                           _ptr(ops["agg"], torch.float64, "agg", dv))
        tot = Totals()
        if op_of_kernel is not None:
            rng = Ranges(None, None, None, None, _ptr(op_of_kernel, torch.uint32, "op_of_kernel", dv), tr.K)
            rok_ptr = None
        else:
            rng = self.ranges(tr)
            rok_ptr = _ptr(range_of_kernel, torch.int32, "range_of_kernel", dv)
        st = opattr_aggregate(self.handle, self.kernels(tr), rng, rok_ptr, self.ncu(tr),
                              _ptr(ncu_idx, torch.int32, "ncu_idx_of_kernel", dv), tr.n_ops, out, tot)
        if st < 0:
            raise OpattrError(st, "opattr_aggregate")
        return st, ops, tot.as_dict()

    def rollup(self, tr: DeviceTrace, range_of_kernel, ncu_idx, class_of_op, n_classes: int, out=None,
               op_of_kernel=None):
        """Per-class records (opattr_rollup); class_of_op: int32/uint32 device tensor of n_ops entries."""
        torch = _torch()
        if out is None:
            out = self.alloc_ops(n_classes)
        dv = self.device
        o = OpAggregates(_ptr(out["kernel_count"], torch.int64, "kernel_count", dv),
                         _ptr(out["total_duration_ns"], torch.int64, "total_duration_ns", dv),
                         _ptr(out["matched_count"], torch.int64, "matched_count", dv),
                         _ptr(out["agg"], torch.float64, "agg", dv))
        if op_of_kernel is not None:
            rng = Ranges(None, None, None, None, _ptr(op_of_kernel, torch.uint32, "op_of_kernel", dv), tr.K)
            rok_ptr = None
        else:
            rng = self.ranges(tr)
            rok_ptr = _ptr(range_of_kernel, torch.int32, "range_of_kernel", dv)
        st = opattr_rollup(self.handle, self.kernels(tr), rng, rok_ptr, self.ncu(tr),
                           _ptr(ncu_idx, torch.int32, "ncu_idx_of_kernel", dv), tr.n_ops,
                           _ptr(class_of_op, torch.uint32, "class_of_op", dv), n_classes, o)
        if st < 0:
            raise OpattrError(st, "opattr_rollup")
        return st, out

    def run(self, tr: DeviceTrace, dedup: bool | None = None):
        """enclose + match + aggregate on device-resident inputs."""
        st_e, rk, nop = self.enclose(tr)
        st_m, idx, kind, summ = self.match(tr, dedup=dedup)
        st_a, ops, tot = self.aggregate(tr, rk, idx)
        return dict(enclose_status=st_e, range_of_kernel=rk, n_op_enclosing=nop, match_status=st_m, ncu_idx=idx,
                    match_kind=kind, summary=summ, aggregate_status=st_a, ops=ops, totals=tot)

    # -- attention, and the paged cache under it.  These calls do not wait; on
    # another stream than the context's they are ordered as calls on that stream
    def _enter(self):
        if _torch()._C._cuda_getCurrentRawStream(self.device) == self._raw_stream:
            return None
        cur = _torch().cuda.current_stream(self.device)
        self.stream.wait_stream(cur)
        return cur

    def _leave(self, cur, status: int, call: str) -> int:
        if cur is not None:
            cur.wait_stream(self.stream)
        if status < 0:
            raise OpattrError(status, call)
        return status

    def _i32(self, t, n: int | None, name):
        if t is None:
            return 0
        shape = t.shape
        if len(shape) != 1 or (n is not None and shape[0] != n):
            raise ValueError(f"{name}: expected [{n if n is not None else 'n'}], got {list(shape)}")
        return _ptr(t, _torch().int32, name, self.device) or 0

    def attention(self, q, k, v, q_offsets=None, k_offsets=None, causal: bool = True, scale: float | None = None,
                  out=None, need_lse: bool = False):
        """Attention over packed sequences (opattr_attention): q [tokens, heads,
        dim], k and v [tokens, kv_heads, dim]; offsets int32 [n_seqs + 1] on the
        device (none: one sequence; k_offsets none: q_offsets).  scale: by
        default 1 / sqrt(dim).  No backward pass: inputs that require a gradient
        are refused where gradients are recorded.  Returns (status, out, lse or None)."""
        torch = _torch()
        dv = self.device
        qs, ks = q.shape, k.shape
        if len(qs) != 3 or len(ks) != 3:
            raise ValueError("q, k: expected [tokens, heads, dim]")
        tokens, heads, dim = qs
        k_tokens, kv_heads, _ = ks
        dt = q.dtype
        dtype = _dtype(q, "q")
        if dim < 8 or dim > 128 or dim % 8:
            raise ValueError(f"dim: expected a multiple of 8 from 8 to 128, got {dim}")
        if kv_heads < 1 or heads < 1 or heads % kv_heads:
            raise ValueError(f"heads: {heads} of q are no multiple of {kv_heads} of k")
        if v.shape[0] != k_tokens:
            raise ValueError(f"v: expected {k_tokens} rows, got {v.shape[0]}")
        if q.requires_grad or k.requires_grad or v.requires_grad:
            _no_grad(q=q, k=k, v=v)
        rq, rk, rv = _rows(q, heads, dim, dt, "q", dv), _rows(k, kv_heads, dim, dt, "k", dv), _rows(v, kv_heads, dim, dt, "v", dv)
        if q_offsets is None:
            if k_offsets is not None:
                raise ValueError("k_offsets: needs q_offsets")
            q_offsets = self._ends(tokens)
            if k_tokens != tokens:
                k_offsets = self._ends(k_tokens)
        n_seqs = q_offsets.numel() - 1
        if n_seqs < 0:
            raise ValueError("q_offsets: expected [n_seqs + 1]")
        if k_offsets is None and k_tokens != tokens:
            raise ValueError("k_offsets: k has other rows than q")
        out, ro = self._out(out, q, heads, dim, dt)
        lse, p_lse = None, 0
        if need_lse:
            lse = torch.empty((tokens, heads), dtype=torch.float32, device=self._dev)
            p_lse = lse.data_ptr()
        p_qo = p_ko = self._i32(q_offsets, n_seqs + 1, "q_offsets")
        if k_offsets is not None and k_offsets is not q_offsets:
            p_ko = self._i32(k_offsets, n_seqs + 1, "k_offsets")
        args = _PROMPT.pack(dtype, n_seqs, heads, kv_heads, dim, 1 if causal else 0, dim ** -0.5 if scale is None else scale,
                            0, tokens, k_tokens, *rq, *rk, *rv, *ro, p_qo, p_ko, p_lse)
        cur = self._enter()
        return self._leave(cur, opattr_attention(self.handle, args), "opattr_attention"), out, lse

    def _ends(self, tokens: int):
        """Offsets of one sequence, made on the device: a copy of host values would wait for it."""
        torch = _torch()
        if tokens == 0:
            return torch.zeros(2, dtype=torch.int32, device=self._dev)
        return torch.arange(0, tokens + 1, tokens, dtype=torch.int32, device=self._dev)

    def _out(self, out, q, heads, dim, dt):
        """An output of q's shape, and its rows."""
        if out is None:
            torch = _torch()
            out = torch.empty_like(q) if q.is_contiguous() else torch.empty(q.shape, dtype=dt, device=self._dev)
            return out, (out.data_ptr(), heads * dim, dim)
        if out.shape != q.shape:
            raise ValueError(f"out: expected {list(q.shape)}, got {list(out.shape)}")
        _distinct(out, "out")
        return out, _rows(out, heads, dim, dt, "out", self.device)

    def cache(self, n_pages: int, page_size: int, kv_heads: int, head_dim: int, n_seqs: int, pages_per_seq: int,
              dtype=None) -> KVCache:
        """An empty cache of `n_pages` pages for `n_seqs` sequences of at most
        pages_per_seq pages each (dtype: by default torch.bfloat16)."""
        torch = _torch()
        new = lambda shape, value: torch.full(shape, value, dtype=torch.int32, device=self._dev)  # noqa: E731
        pool = [torch.zeros((n_pages, kv_heads, page_size, head_dim), dtype=dtype or torch.bfloat16, device=self._dev)
                for _ in range(2)]
        return KVCache(*pool, new((n_seqs, pages_per_seq), -1), new((n_seqs,), 0), new((n_pages,), 0), new((1,), 0))

    def _cache(self, cache: KVCache) -> Cache:
        if cache.device != self.device:
            raise ValueError(f"cache: must live on cuda:{self.device}")
        return cache.struct

    def cache_attention(self, cache: KVCache, seqs, q, scale: float | None = None, out=None, need_lse: bool = False):
        """Attention of one new token per sequence over the cache
        (opattr_cache_attention): q [n, heads, dim], row i of sequence seqs[i]
        (int32 [n], or None: sequence i).  Returns (status, out, lse or None)."""
        torch = _torch()
        kv = self._cache(cache)
        dim, dt = kv.head_dim, cache.k_pages.dtype
        rq = _rows(q, None, dim, dt, "q", self.device)
        n, heads, _ = q.shape
        if heads < 1 or heads % kv.kv_heads:
            raise ValueError(f"heads: {heads} of q are no multiple of {kv.kv_heads} of the cache")
        if seqs is None and n > kv.n_seqs:
            raise ValueError(f"q: {n} rows for {kv.n_seqs} sequences")
        if q.requires_grad:
            _no_grad(q=q)
        out, ro = self._out(out, q, heads, dim, dt)
        lse, p_lse = None, 0
        if need_lse:
            lse = torch.empty((n, heads), dtype=torch.float32, device=self._dev)
            p_lse = lse.data_ptr()
        p_seqs = self._i32(seqs, n, "seqs")
        cur = self._enter()
        st = opattr_cache_attention(self.handle, cache.by_ref, p_seqs, n, heads, _ROWS.pack(*rq), _ROWS.pack(*ro), p_lse, dim ** -0.5 if scale is None else scale)
        return self._leave(cur, st, "opattr_cache_attention"), out, lse

    def cache_append(self, cache: KVCache, seqs, offsets, k, v) -> int:
        """Rows offsets[i] .. offsets[i + 1] of k and v ([tokens, kv_heads, dim])
        to the end of sequence seqs[i], each sequence once (opattr_cache_append)."""
        kv = self._cache(cache)
        if v.shape != k.shape:
            raise ValueError(f"v: expected {list(k.shape)}, got {list(v.shape)}")
        if k.requires_grad or v.requires_grad:
            _no_grad(k=k, v=v)
        dt = cache.k_pages.dtype
        rk = _rows(k, kv.kv_heads, kv.head_dim, dt, "k", self.device)
        rv = _rows(v, kv.kv_heads, kv.head_dim, dt, "v", self.device)
        p_seqs = self._i32(seqs, None, "seqs")
        n = seqs.shape[0]
        p_off = self._i32(offsets, n + 1, "offsets")
        cur = self._enter()
        st = opattr_cache_append(self.handle, cache.by_ref, p_seqs, n, p_off, k.shape[0],
                                 _ROWS.pack(*rk), _ROWS.pack(*rv))
        return self._leave(cur, st, "opattr_cache_append")

    def cache_fork(self, cache: KVCache, src, dst) -> int:
        """The empty sequences dst[i] share the pages of src[i] (opattr_cache_fork)."""
        self._cache(cache)
        p_dst = self._i32(dst, None, "dst")
        n = dst.shape[0]
        p_src = self._i32(src, n, "src")
        cur = self._enter()
        return self._leave(cur, opattr_cache_fork(self.handle, cache.by_ref, p_src, p_dst, n), "opattr_cache_fork")

    def cache_trim(self, cache: KVCache, seqs, lengths=None) -> int:
        """Sequence seqs[i] keeps its first lengths[i] tokens (none: it is
        freed), and the pages past them are let go (opattr_cache_trim)."""
        self._cache(cache)
        p_seqs = self._i32(seqs, None, "seqs")
        n = seqs.shape[0]
        p_len = self._i32(lengths, n, "lengths")
        cur = self._enter()
        return self._leave(cur, opattr_cache_trim(self.handle, cache.by_ref, p_seqs, p_len, n), "opattr_cache_trim")

    def cache_compact(self, cache: KVCache):
        """The pages in use become the cache's first ones (opattr_cache_compact).
        Returns (status, int32 [1] tensor of how many those are)."""
        torch = _torch()
        self._cache(cache)
        live = torch.empty(1, dtype=torch.int32, device=self._dev)
        cur = self._enter()
        st = opattr_cache_compact(self.handle, cache.by_ref, live.data_ptr())
        return self._leave(cur, st, "opattr_cache_compact"), live

    def check(self) -> None:
        """Waits for the calls above and raises what they found wrong on the
        device since the last check (opattr_check)."""
        st = opattr_check(self.handle)
        if st < 0:
            raise OpattrError(st, "opattr_check")

    # -- accounting
    def set_timing(self, on: bool):
        library().opattr_set_timing(self.handle, int(bool(on)))

    def set_timing_only(self, kernel: str | None):
        """With timing on, bracket only the launches of `kernel` (None: all)."""
        library().opattr_set_timing_only(self.handle, kernel.encode() if kernel else None)

    def timing_report(self) -> dict:
        lib = library()
        n = lib.opattr_timing_report(self.handle, None, None, None, 0)
        names = (ctypes.c_char_p * max(n, 1))()
        ms = (ctypes.c_double * max(n, 1))()
        cnt = (ctypes.c_int64 * max(n, 1))()
        lib.opattr_timing_report(self.handle, names, ms, cnt, n)
        return {names[i].decode(): (float(ms[i]), int(cnt[i])) for i in range(n)}

    def timing_reset(self):
        library().opattr_timing_reset(self.handle)

    def launch_count(self) -> int:
        return int(library().opattr_launch_count(self.handle))
