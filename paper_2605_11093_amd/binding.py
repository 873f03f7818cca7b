"""ctypes binding of include/dmi.h, include/dmi_kv8.h and include/dmi_kv8_long.h: same names, argument marshalling only.

Every step of the capture-and-stage path runs inside libdmi.so.  There is no
fallback: if the library is missing or no GPU is present the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import sys
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np

try:                        # native marshalling of the per-tensor calls; without it they go through ctypes
    from . import _dmi_python as _native
    if getattr(_native, "INTERFACE", 0) != 2:       # (built from other sources, and about to be built again)
        _native = None
except ImportError:
    _native = None

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "libdmi.so")
_lib = None

OK, SAMPLED_OUT, POINT_DISABLED = 0, 1, 2
ERR_INVALID_ARG, ERR_NOMEM, ERR_TOO_LARGE, ERR_HIP, ERR_AGAIN, ERR_CLOSED = -1, -2, -3, -4, -5, -6
DT_NONE, DT_BF16, DT_FP16, DT_FP32, DT_FP8 = 0, 1, 2, 3, 4
SUM_L2, SUM_MEAN, SUM_ABSMAX = 1, 2, 4
POLICY_BLOCK, POLICY_DROP_NEWEST = 0, 1
DRAIN_COPY_ENGINE, DRAIN_KERNEL, BG_THREAD = 1, 2, 4
DRAIN_NONBLOCK, DRAIN_FLUSH = 1, 2


class DmiError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"dmi error {code}: {msg}")
        self.code = code


class RingConfig(C.Structure):
    _fields_ = [("device_ring_bytes", C.c_uint64), ("host_ring_bytes", C.c_uint64),
                ("device_id", C.c_int32), ("flags", C.c_uint32),
                ("max_reqs_per_observe", C.c_uint32), ("rank_tag", C.c_uint32),
                ("bg_min_bytes", C.c_uint64), ("bg_timeout_us", C.c_uint32),
                ("block_timeout_ms", C.c_uint32), ("bg_min_records", C.c_uint32),
                ("bg_occupancy_pct", C.c_uint32)]


class Tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_uint32), ("shape", C.c_int64 * 2),
                ("stride", C.c_int64 * 2)]


class ReqSel(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("req_id", "row_base", "tok_start", "tok_count", "tok_step")]


class Selection(C.Structure):
    _fields_ = [("n_reqs", C.c_uint32), ("reqs", C.c_void_p), ("keep_mask_dev", C.c_void_p),
                ("row_index_dev", C.c_void_p)]


class Transform(C.Structure):
    _fields_ = [("out_dtype", C.c_uint32), ("summary_mask", C.c_uint32)]


class PagedKV(C.Structure):
    _fields_ = [("base", C.c_void_p), ("dtype", C.c_uint32), ("block_stride", C.c_int64),
                ("slot_stride", C.c_int64), ("head_stride", C.c_int64),
                ("block_size", C.c_uint32), ("n_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("n_blocks", C.c_uint32), ("n_seqs", C.c_uint32),
                ("block_table_dev", C.c_void_p), ("block_table_stride", C.c_int64),
                ("n_heads_sel", C.c_uint32), ("heads_sel", C.c_uint32 * 8)]


class RecordViewC(C.Structure):
    _fields_ = [("p0", C.c_void_p), ("n0", C.c_uint64), ("p1", C.c_void_p), ("n1", C.c_uint64),
                ("seq", C.c_uint64)]


class ReqInfo(C.Structure):
    _fields_ = [("req_id", C.c_uint32), ("rows", C.c_uint32), ("admit_order", C.c_uint64),
                ("matches", C.c_uint32), ("reserved", C.c_uint32)]


class SliceC(C.Structure):
    _fields_ = [("seq", C.c_uint64), ("step_id", C.c_uint64), ("point_id", C.c_uint32), ("rank_tag", C.c_uint32),
                ("req_index", C.c_uint32), ("req_id", C.c_uint32), ("tok_start", C.c_uint32),
                ("tok_step", C.c_uint32), ("n_rows", C.c_uint32), ("row_elems", C.c_uint32),
                ("src_dtype", C.c_uint32), ("out_dtype", C.c_uint32), ("summary_mask", C.c_uint32),
                ("flags", C.c_uint32), ("rows", C.c_void_p), ("l2", C.c_void_p), ("mean", C.c_void_p),
                ("absmax", C.c_void_p), ("owner", C.c_void_p)]


class Policy(C.Structure):
    _fields_ = [("mode", C.c_uint32), ("sample_k", C.c_uint32), ("sample_phase", C.c_uint32)]


_STAT_FIELDS = ("observed_calls", "launched_records", "captured_records", "captured_rows",
                "captured_bytes", "dropped_records", "dropped_rows", "dropped_bytes",
                "sampled_out_calls", "sampled_out_rows", "disabled_calls", "drained_bytes",
                "released_bytes", "drain_batches", "block_wait_ns", "dev_ring_high_water",
                "host_ring_high_water", "bad_rows")


class StatsC(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in _STAT_FIELDS]


@dataclass
class Stats:
    observed_calls: int = 0
    launched_records: int = 0
    captured_records: int = 0
    captured_rows: int = 0
    captured_bytes: int = 0
    dropped_records: int = 0
    dropped_rows: int = 0
    dropped_bytes: int = 0
    sampled_out_calls: int = 0
    sampled_out_rows: int = 0
    disabled_calls: int = 0
    drained_bytes: int = 0
    released_bytes: int = 0
    drain_batches: int = 0
    block_wait_ns: int = 0
    dev_ring_high_water: int = 0
    host_ring_high_water: int = 0
    bad_rows: int = 0


@dataclass
class RecordView:
    seq: int
    p0: int
    n0: int
    p1: int
    n1: int

    @property
    def nbytes(self) -> int:
        return self.n0 + self.n1

    def bytes(self) -> np.ndarray:
        """Copy of the record's bytes (valid only until the record is released)."""
        out = np.empty(self.n0 + self.n1, dtype=np.uint8)
        C.memmove(out.ctypes.data, self.p0, self.n0)
        if self.n1:
            C.memmove(out.ctypes.data + self.n0, self.p1, self.n1)
        return out


def library_path() -> str:
    return _SO


def lib():
    """Load libdmi.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_SO):
        raise ImportError(f"{_SO} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
    L = C.CDLL(_SO)
    P = C.POINTER
    L.dmi_last_error.restype = C.c_char_p
    L.dmi_version.restype = C.c_char_p
    L.dmi_record_bytes.restype = C.c_uint64
    L.dmi_record_bytes.argtypes = [C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32]
    L.dmi_ring_create.argtypes = [P(RingConfig), P(C.c_void_p)]
    L.dmi_ring_destroy.argtypes = [C.c_void_p]
    L.dmi_observe.argtypes = [C.c_void_p, C.c_uint32, P(Tensor), P(Selection), P(Transform),
                              C.c_uint64, C.c_void_p]
    L.dmi_observe_paged.argtypes = [C.c_void_p, C.c_uint32, P(PagedKV), P(Selection), P(Transform),
                                    C.c_uint64, C.c_void_p]
    L.dmi_observe_batch.argtypes = [C.c_void_p, C.c_uint32, P(C.c_uint32), P(C.c_void_p), P(Tensor), P(Selection),
                                    P(Transform), C.c_uint64, C.c_void_p, P(C.c_uint32)]
    L.dmi_observe_paged_batch.argtypes = [C.c_void_p, C.c_uint32, P(C.c_uint32), P(C.c_void_p), P(PagedKV),
                                          P(Selection), P(Transform), C.c_uint64, C.c_void_p, P(C.c_uint32)]
    L.dmi_step_observe_batch.argtypes = [C.c_void_p, C.c_uint32, P(C.c_uint32), P(C.c_void_p), P(Tensor),
                                         P(Selection), P(Transform), C.c_void_p, P(C.c_uint32)]
    L.dmi_step_observe_paged_batch.argtypes = [C.c_void_p, C.c_uint32, P(C.c_uint32), P(C.c_void_p), P(PagedKV),
                                               P(Selection), P(Transform), C.c_void_p, P(C.c_uint32)]
    for name in ("dmi_observe_batch", "dmi_observe_paged_batch", "dmi_step_observe_batch",
                 "dmi_step_observe_paged_batch"):
        getattr(L, name).restype = C.c_int32
    L.dmi_observe_into.argtypes = [C.c_uint32, P(Tensor), P(Selection), P(Transform), C.c_uint64, C.c_uint64,
                                   C.c_uint32, C.c_void_p, C.c_uint64, P(C.c_uint64), C.c_void_p]
    L.dmi_observe_into.restype = C.c_int32
    # (the structs of dmi_kv8.h go as bytes: see KV8)
    S = C.c_char_p
    L.dmi_kv8_append.argtypes = [S, S, S, S, C.c_void_p]
    L.dmi_kv8_attend_workspace.argtypes = [S, S, C.c_uint32, C.c_int]
    L.dmi_kv8_attend_workspace.restype = C.c_uint64
    L.dmi_kv8_attend.argtypes = [S, S, S, C.c_uint32, C.c_float, S, C.c_void_p, S, S, C.c_float, C.c_void_p, C.c_uint64,
                                 C.c_void_p]
    L.dmi_kv8_evict.argtypes = [S, S, S, S, S, C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p]
    L.dmi_kv8_append_rotated.argtypes = [S, S, S, S, S, S, C.c_uint32, S, C.c_void_p]
    L.dmi_kv8_bound.argtypes = [S, S, S, C.c_void_p]
    L.dmi_kv8_select_workspace.argtypes = [S, S, C.c_uint32]
    L.dmi_kv8_select.argtypes = [S, S, S, S, C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
    L.dmi_kv8_attend_blocks_workspace.argtypes = [S, S, C.c_uint32, C.c_uint32]
    L.dmi_kv8_attend_blocks.argtypes = [S, S, C.c_void_p, C.c_uint32, S, C.c_uint32, C.c_float, S, C.c_void_p, C.c_void_p, C.c_uint64,
                                        C.c_void_p]
    L.dmi_kv8_attend_shared_workspace.argtypes = [S, S, S, C.c_uint32]
    L.dmi_kv8_attend_shared.argtypes = [S, S, S, S, C.c_uint32, C.c_float, S, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
    for name in ("select", "attend_blocks", "attend_shared"):
        getattr(L, f"dmi_kv8_{name}_workspace").restype = C.c_uint64
    for name in ("dmi_kv8_append", "dmi_kv8_attend", "dmi_kv8_evict", "dmi_kv8_append_rotated", "dmi_kv8_bound", "dmi_kv8_select",
                 "dmi_kv8_attend_blocks", "dmi_kv8_attend_shared"):
        getattr(L, name).restype = C.c_int32
    L.dmi_drain.argtypes = [C.c_void_p, C.c_uint32, P(C.c_uint64)]
    L.dmi_poll_host.argtypes = [C.c_void_p, P(RecordViewC), C.c_uint32, P(C.c_uint32)]
    L.dmi_release_host.argtypes = [C.c_void_p, C.c_uint64]
    L.dmi_set_policy.argtypes = [C.c_void_p, P(Policy)]
    L.dmi_point_enable.argtypes = [C.c_void_p, C.c_uint32, C.c_int]
    L.dmi_get_stats.argtypes = [C.c_void_p, P(StatsC)]
    L.dmi_get_point_drops.argtypes = [C.c_void_p, C.c_uint32, P(C.c_uint64)]
    L.dmi_debug_fill_rings.argtypes = [C.c_void_p, C.c_uint8]
    L.dmi_debug_exporter_allocs.argtypes = [C.c_void_p, P(C.c_uint64), P(C.c_uint64)]
    L.dmi_debug_exporter_allocs.restype = C.c_int32
    L.dmi_debug_time_next_launch.argtypes = [C.c_void_p, C.c_void_p]
    L.dmi_debug_time_next_launch.restype = C.c_int32
    L.dmi_exporter_start.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32]
    L.dmi_exporter_next.argtypes = [C.c_void_p, P(SliceC), C.c_uint32]
    L.dmi_exporter_release.argtypes = [C.c_void_p, P(SliceC)]
    L.dmi_exporter_next_many.argtypes = [C.c_void_p, P(SliceC), C.c_uint32, P(C.c_uint32), C.c_uint32]
    L.dmi_exporter_release_many.argtypes = [C.c_void_p, P(SliceC), C.c_uint32]
    L.dmi_exporter_stop.argtypes = [C.c_void_p]
    L.dmi_policy_select.argtypes = [C.c_uint32, P(ReqInfo), C.c_uint32, C.c_uint64, C.c_uint64, C.c_void_p,
                                    P(C.c_uint32)]
    L.dmi_ring_free_bytes.argtypes = [C.c_void_p, P(C.c_uint64)]
    L.dmi_set_keep_mask.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32, C.c_void_p, P(C.c_void_p)]
    L.dmi_step_create.argtypes = [C.c_void_p, C.c_uint32, P(C.c_void_p)]
    L.dmi_step_destroy.argtypes = [C.c_void_p]
    L.dmi_step_capture_begin.argtypes = [C.c_void_p]
    L.dmi_step_observe.argtypes = [C.c_void_p, C.c_uint32, P(Tensor), P(Selection), P(Transform), C.c_void_p,
                                   P(C.c_uint32)]
    L.dmi_step_observe_paged.argtypes = [C.c_void_p, C.c_uint32, P(PagedKV), P(Selection), P(Transform),
                                         C.c_void_p, P(C.c_uint32)]
    L.dmi_step_seal.argtypes = [C.c_void_p]
    L.dmi_step_update.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p, C.c_uint32]
    L.dmi_step_begin.argtypes = [C.c_void_p, C.c_uint64, C.c_void_p]
    L.dmi_step_end.argtypes = [C.c_void_p, C.c_void_p]
    for name in ("dmi_step_create", "dmi_step_destroy", "dmi_step_capture_begin", "dmi_step_observe",
                 "dmi_step_observe_paged", "dmi_step_seal", "dmi_step_update", "dmi_step_begin", "dmi_step_end"):
        getattr(L, name).restype = C.c_int32
    for name in ("dmi_ring_create", "dmi_ring_destroy", "dmi_observe", "dmi_observe_paged", "dmi_drain",
                 "dmi_poll_host", "dmi_release_host", "dmi_set_policy", "dmi_point_enable",
                 "dmi_get_stats", "dmi_get_point_drops", "dmi_debug_fill_rings", "dmi_policy_select",
                 "dmi_ring_free_bytes", "dmi_set_keep_mask", "dmi_exporter_start", "dmi_exporter_next",
                 "dmi_exporter_release", "dmi_exporter_stop", "dmi_exporter_next_many",
                 "dmi_exporter_release_many"):
        getattr(L, name).restype = C.c_int32
    _lib = L
    if _native is not None:
        _native_calls(L)
    return L


_reader_asked = False
_native_ok = False          # the native modules were built with the library's dmi.h


def _native_calls(L):
    """The library's entry points for the native modules, if the structs they hand over are the library's."""
    global _native_ok
    try:
        L.dmi_debug_header_digest.restype = C.c_uint64
        _native_ok = L.dmi_debug_header_digest() == _native.HEADER_DIGEST
    except AttributeError:                          # (an older library)
        _native_ok = False
    if _native_ok:
        _load_reader()
        _native.bind_into(C.cast(L.dmi_observe_into, C.c_void_p).value)


def _load_reader():
    """The native module that reads tensors, once, as soon as torch is there: a library that a process loads with its GPU in use already
    costs every later launch 0.2 us."""
    global _reader_asked
    if _reader_asked or _native is None or "torch" not in sys.modules:
        return
    _reader_asked = True
    try:
        from . import _dmi_python_torch
        _native.set_reader(_dmi_python_torch.reader)
    except Exception:                               # (another torch than it was built for: ctypes does)
        pass


def version() -> str:
    return lib().dmi_version().decode()


def record_bytes(n_reqs: int, n_rows: int, row_elems: int, out_dtype: int, summary_mask: int) -> int:
    return int(lib().dmi_record_bytes(n_reqs, n_rows, row_elems, out_dtype, summary_mask))


SELECT_DROP_RECENT, SELECT_KEEP_BY_PATTERN = 0, 1


def policy_select(strategy: int, reqs, bytes_per_row: int, budget_bytes: int) -> np.ndarray:
    """reqs: iterable of (req_id, rows, admit_order, matches).  Returns the keep vector (uint8)."""
    rows = list(reqs)
    arr = (ReqInfo * max(1, len(rows)))(*[ReqInfo(int(a), int(b), int(c), int(d), 0) for a, b, c, d in rows])
    keep = np.zeros(len(rows), dtype=np.uint8)
    n = C.c_uint32()
    _check(lib().dmi_policy_select(strategy, arr, len(rows), bytes_per_row, budget_bytes,
                                   keep.ctypes.data if len(rows) else None, C.byref(n)))
    assert int(n.value) == int(keep.sum())
    return keep


def _check(code: int, allow: Sequence[int] = ()) -> int:
    if code < 0 and code not in allow:
        raise DmiError(code, lib().dmi_last_error().decode())
    return code


_TORCH_DT = None


def _torch_dtype_code(t) -> int:
    global _TORCH_DT
    if _TORCH_DT is None:
        import torch
        _TORCH_DT = {torch.bfloat16: DT_BF16, torch.float16: DT_FP16, torch.float32: DT_FP32}
    return _TORCH_DT[t.dtype]


def time_next_launch(start_event: int, stop_event: int) -> None:
    """The calling thread's next capture launch records its own start and end into the two hipEvent_t handles."""
    _check(lib().dmi_debug_time_next_launch(start_event or None, stop_event or None))


def _reqs_buffer(reqs):
    a = np.ascontiguousarray(np.asarray(reqs, dtype=np.uint32).reshape(-1, 5))
    return a


# dmi_tensor_t, dmi_selection_t and dmi_transform_t as bytes (the structs above, padding included)
_PACK_TENSOR = struct.Struct("=QI4xqqqq").pack
_PACK_SELECTION = struct.Struct("=I4xQQQ").pack
_PACK_TRANSFORM = struct.Struct("=II").pack
_into_fn = None             # set: what observe_into calls in place of the library's entry point, structs as bytes
_into_bytes = None


def _into_raw():
    """dmi_observe_into taking its structs as bytes."""
    global _into_bytes
    if _into_fn is not None:
        return _into_fn
    if _into_bytes is None:
        f = lib()["dmi_observe_into"]
        f.restype = C.c_int32
        f.argtypes = [C.c_uint32, C.c_char_p, C.c_char_p, C.c_char_p, C.c_uint64, C.c_uint64, C.c_uint32, C.c_void_p,
                      C.c_uint64, C.c_void_p, C.c_void_p]
        _into_bytes = f
    return _into_bytes


def observe_into(point_id: int, tensor, reqs, out, *, seq: int, step_id: int, rank_tag: int = 0,
                 out_dtype: Optional[int] = None, summary_mask: int = 0, keep_mask=None, row_index=None,
                 stream: int = 0, allow: Sequence[int] = ()) -> int:
    """dmi_observe_into: one record into `out` (a uint8 device tensor), no ring, no allocation.
    Returns the record's size (an upper bound if a keep vector is given)."""
    dt = _torch_dtype_code(tensor)
    shape = tensor.shape
    if type(reqs) is not np.ndarray or reqs.dtype != np.uint32 or reqs.ndim != 2 or reqs.shape[1] != 5 \
            or not reqs.flags.c_contiguous:
        reqs = _reqs_buffer(reqs)
    # A small capture takes the GPU a few microseconds, and building the three argument structs as ctypes objects took
    # longer than that (8.2 us a call, 4 us like this): they are packed into bytes of the same layout.
    stride = tensor.stride()
    if len(shape) != 2:                             # the ABI refuses a row length of 0
        if len(shape) > 2:
            raise IndexError("invalid index: observe_into takes a matrix")
        shape, stride = (*shape, 0, 0)[:2], (*stride, 0, 0)[:2]
    t = _PACK_TENSOR(tensor.data_ptr(), dt, shape[0], shape[1], stride[0], stride[1])
    try:
        at = C.addressof(C.c_char.from_buffer(reqs))
    except (TypeError, ValueError):                 # read-only, or empty
        at = reqs.ctypes.data
    sel = _PACK_SELECTION(len(reqs), at, 0 if keep_mask is None else keep_mask.data_ptr(),
                          0 if row_index is None else row_index.data_ptr())
    xf = _PACK_TRANSFORM((dt if out_dtype is None else out_dtype) & 0xFFFFFFFF, summary_mask & 0xFFFFFFFF)
    n = C.c_uint64()
    _check(_into_raw()(point_id, t, sel, xf, seq, step_id, rank_tag, out.data_ptr(), out.numel() * out.element_size(),
                       C.byref(n), stream or None), allow)
    return n.value


if _native is not None:     # the plain case without Python in between; all else comes back to the function above
    _general_into = observe_into
    _native.setup(_general_into, _check, globals(), _load_reader)
    observe_into = _native.observe_into
    _load_reader()


class PreparedObserve(_native.Prepared if _native is not None else object):
    """The argument structs of one dmi_observe / dmi_observe_paged call, built once so
    that a per-step loop pays only the foreign call itself.  Calling it returns the
    raw status code."""

    def __init__(self, ring: "Ring", point_id: int, tensor, reqs, *, out_dtype: Optional[int] = None,
                 summary_mask: int = 0, keep_mask=None, row_index=None, paged=None):
        dt = _torch_dtype_code(tensor)
        self._keep = (tensor, keep_mask, row_index, paged)
        self._ra = _reqs_buffer(reqs)
        self._sel = Selection(self._ra.shape[0], self._ra.ctypes.data,
                              None if keep_mask is None else keep_mask.data_ptr(),
                              None if row_index is None else row_index.data_ptr())
        self._xf = Transform(dt if out_dtype is None else out_dtype, summary_mask)
        self._h, self._point = ring._h, point_id
        if paged is None:
            self._src = Tensor(tensor.data_ptr(), dt, (C.c_int64 * 2)(*tensor.shape),
                               (C.c_int64 * 2)(*tensor.stride()))
            self._fn = lib().dmi_observe
        else:
            bt = paged.block_table
            self._src = PagedKV(tensor.data_ptr(), dt, tensor.stride(0), tensor.stride(1), tensor.stride(2),
                                paged.block_size, paged.n_heads, paged.head_dim, tensor.shape[0], bt.shape[0],
                                bt.data_ptr(), bt.stride(0), len(paged.heads_sel),
                                (C.c_uint32 * 8)(*paged.heads_sel))
            self._fn = lib().dmi_observe_paged
        self._a = (C.byref(self._src), C.byref(self._sel), C.byref(self._xf))
        if _native_ok and type(point_id) is int and self._h:
            self._bind(C.cast(self._fn, C.c_void_p).value, self._h.value, point_id & 0xFFFFFFFF, C.addressof(self._src),
                       C.addressof(self._sel), C.addressof(self._xf))

    def __getstate__(self):                         # (a copy calls through Python)
        return self.__dict__

    def _call(self, step_id: int, stream: int) -> int:
        return self._fn(self._h, self._point, self._a[0], self._a[1], self._a[2], step_id, stream)

    if _native is None:
        __call__ = _call


def _paged_struct(cache, paged_or_table, *, block_size=None, n_heads=None, head_dim=None, heads_sel=None):
    """dmi_paged_kv_t for a cache tensor [blocks, slots, heads, dim]."""
    if block_size is None:
        p = paged_or_table
        bt, block_size, n_heads, head_dim, heads_sel = p.block_table, p.block_size, p.n_heads, p.head_dim, p.heads_sel
    else:
        bt = paged_or_table
    return PagedKV(cache.data_ptr(), _torch_dtype_code(cache), cache.stride(0), cache.stride(1), cache.stride(2),
                   block_size, n_heads, head_dim, cache.shape[0], bt.shape[0], bt.data_ptr(), bt.stride(0),
                   len(heads_sel), (C.c_uint32 * 8)(*heads_sel))


def _same_layout(tensors):
    t0 = tensors[0]
    for t in tensors[1:]:
        if t.dtype != t0.dtype or tuple(t.shape) != tuple(t0.shape) or tuple(t.stride()) != tuple(t0.stride()):
            raise ValueError("the tensors of a batch must share dtype, shape and strides")


class PreparedBatch:
    """The argument structs of one dmi_observe_batch / dmi_observe_paged_batch call, built once.
    Calling it returns (status, n_done)."""

    def __init__(self, ring: "Ring", point_ids, tensors, reqs, *, out_dtype: Optional[int] = None,
                 summary_mask: int = 0, keep_mask=None, row_index=None, paged=None):
        tensors = list(tensors)
        _same_layout(tensors)
        dt = _torch_dtype_code(tensors[0])
        self._keep = (tensors, keep_mask, row_index, paged)
        self._n = len(tensors)
        self._points = (C.c_uint32 * self._n)(*[int(p) for p in point_ids])
        self._data = (C.c_void_p * self._n)(*[t.data_ptr() for t in tensors])
        self._ra = _reqs_buffer(reqs)
        self._sel = Selection(self._ra.shape[0], self._ra.ctypes.data,
                              None if keep_mask is None else keep_mask.data_ptr(),
                              None if row_index is None else row_index.data_ptr())
        self._xf = Transform(dt if out_dtype is None else out_dtype, summary_mask)
        self._h = ring._h
        t0 = tensors[0]
        if paged is None:
            self._like = Tensor(t0.data_ptr(), dt, (C.c_int64 * 2)(*t0.shape), (C.c_int64 * 2)(*t0.stride()))
            self._fn = lib().dmi_observe_batch
        else:
            self._like = _paged_struct(t0, paged)
            self._fn = lib().dmi_observe_paged_batch
        self._done = C.c_uint32()

    def __call__(self, step_id: int, stream: int):
        rc = self._fn(self._h, self._n, self._points, self._data, C.byref(self._like), C.byref(self._sel),
                      C.byref(self._xf), step_id, stream, C.byref(self._done))
        return rc, self._done.value


class Step:
    """A replayable step (dmi_step_*): capture launches that can sit in a captured graph."""

    def __init__(self, ring: "Ring", max_observes: int):
        h = C.c_void_p()
        _check(lib().dmi_step_create(ring._h, max_observes, C.byref(h)))
        self._h = h
        self._ring = ring

    def destroy(self):
        if self._h:
            _check(lib().dmi_step_destroy(self._h))
            self._h = None

    def capture_begin(self):
        _check(lib().dmi_step_capture_begin(self._h))

    def observe_tensor(self, point_id: int, tensor, reqs, *, stream: int, out_dtype: Optional[int] = None,
                       summary_mask: int = 0, keep_mask=None, row_index=None, allow: Sequence[int] = ()) -> int:
        """Returns the node index, or -1 if the point is disabled (nothing launched)."""
        dt = _torch_dtype_code(tensor)
        ra = _reqs_buffer(reqs)
        t = Tensor(tensor.data_ptr(), dt, (C.c_int64 * 2)(*tensor.shape), (C.c_int64 * 2)(*tensor.stride()))
        sel = Selection(ra.shape[0], ra.ctypes.data, None if keep_mask is None else keep_mask.data_ptr(),
                        None if row_index is None else row_index.data_ptr())
        xf = Transform(dt if out_dtype is None else out_dtype, summary_mask)
        node = C.c_uint32()
        code = _check(lib().dmi_step_observe(self._h, point_id, C.byref(t), C.byref(sel), C.byref(xf),
                                             stream or None, C.byref(node)), allow)
        return int(node.value) if code == OK else -1

    def observe_paged(self, point_id: int, cache, block_table, reqs, *, block_size: int, n_heads: int,
                      head_dim: int, heads_sel: Sequence[int], stream: int, out_dtype: Optional[int] = None,
                      summary_mask: int = 0, keep_mask=None, allow: Sequence[int] = ()) -> int:
        dt = _torch_dtype_code(cache)
        ra = _reqs_buffer(reqs)
        kv = PagedKV(cache.data_ptr(), dt, cache.stride(0), cache.stride(1), cache.stride(2),
                     block_size, n_heads, head_dim, cache.shape[0], block_table.shape[0],
                     block_table.data_ptr(), block_table.stride(0), len(heads_sel),
                     (C.c_uint32 * 8)(*heads_sel))
        sel = Selection(ra.shape[0], ra.ctypes.data, None if keep_mask is None else keep_mask.data_ptr(), None)
        xf = Transform(dt if out_dtype is None else out_dtype, summary_mask)
        node = C.c_uint32()
        code = _check(lib().dmi_step_observe_paged(self._h, point_id, C.byref(kv), C.byref(sel), C.byref(xf),
                                                   stream or None, C.byref(node)), allow)
        return int(node.value) if code == OK else -1

    def observe_batch(self, point_ids, tensors, reqs, *, stream: int, out_dtype: Optional[int] = None,
                      summary_mask: int = 0, keep_mask=None, row_index=None, paged=None,
                      allow: Sequence[int] = ()) -> int:
        """n tensors of one layout -> n consecutive records of the step, one launch.
        Returns the index of the first record, or -1 if every point is disabled."""
        tensors = list(tensors)
        _same_layout(tensors)
        n, t0 = len(tensors), tensors[0]
        dt = _torch_dtype_code(t0)
        ra = _reqs_buffer(reqs)
        pts = (C.c_uint32 * n)(*[int(p) for p in point_ids])
        data = (C.c_void_p * n)(*[t.data_ptr() for t in tensors])
        sel = Selection(ra.shape[0], ra.ctypes.data, None if keep_mask is None else keep_mask.data_ptr(),
                        None if row_index is None else row_index.data_ptr())
        xf = Transform(dt if out_dtype is None else out_dtype, summary_mask)
        node = C.c_uint32()
        if paged is None:
            like = Tensor(t0.data_ptr(), dt, (C.c_int64 * 2)(*t0.shape), (C.c_int64 * 2)(*t0.stride()))
            code = lib().dmi_step_observe_batch(self._h, n, pts, data, C.byref(like), C.byref(sel), C.byref(xf),
                                                stream or None, C.byref(node))
        else:
            like = _paged_struct(t0, paged)
            code = lib().dmi_step_observe_paged_batch(self._h, n, pts, data, C.byref(like), C.byref(sel),
                                                      C.byref(xf), stream or None, C.byref(node))
        _check(code, allow)
        return int(node.value) if code == OK else -1

    def seal(self):
        _check(lib().dmi_step_seal(self._h))

    def update(self, node: int, reqs, allow: Sequence[int] = ()) -> int:
        ra = _reqs_buffer(reqs)
        return _check(lib().dmi_step_update(self._h, node, ra.ctypes.data, ra.shape[0]), allow)

    def begin(self, step_id: int, stream: int, allow: Sequence[int] = ()) -> int:
        return _check(lib().dmi_step_begin(self._h, step_id, stream or None), allow)

    def end(self, stream: int) -> int:
        return _check(lib().dmi_step_end(self._h, stream or None))


class Ring:
    """Thin object wrapper: one method per C entry point."""

    def __init__(self, device_ring_bytes: int, host_ring_bytes: int, *, device_id: int = 0,
                 flags: int = 0, max_reqs_per_observe: int = 0, rank_tag: int = 0,
                 bg_min_bytes: int = 0, bg_timeout_us: int = 0, block_timeout_ms: int = 0,
                 bg_min_records: int = 0, bg_occupancy_pct: int = 0):
        cfg = RingConfig(device_ring_bytes, host_ring_bytes, device_id, flags, max_reqs_per_observe,
                         rank_tag, bg_min_bytes, bg_timeout_us, block_timeout_ms, bg_min_records,
                         bg_occupancy_pct)
        h = C.c_void_p()
        _check(lib().dmi_ring_create(C.byref(cfg), C.byref(h)))
        self._h = h
        self._views = (RecordViewC * 256)()

    # -- lifetime --------------------------------------------------------
    def destroy(self):
        if self._h:
            _check(lib().dmi_ring_destroy(self._h))
            self._h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.destroy()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # -- producer --------------------------------------------------------
    def observe(self, point_id: int, data_ptr: int, dtype: int, shape, stride, reqs, *,
                step_id: int, stream: int = 0, out_dtype: int = DT_BF16, summary_mask: int = 0,
                keep_mask_dev: int = 0, row_index_dev: int = 0, allow: Sequence[int] = ()) -> int:
        ra = _reqs_buffer(reqs)
        t = Tensor(data_ptr, dtype, (C.c_int64 * 2)(*shape), (C.c_int64 * 2)(*stride))
        sel = Selection(ra.shape[0], ra.ctypes.data, keep_mask_dev or None, row_index_dev or None)
        xf = Transform(out_dtype, summary_mask)
        return _check(lib().dmi_observe(self._h, point_id, C.byref(t), C.byref(sel), C.byref(xf),
                                        step_id, stream or None), allow)

    def observe_tensor(self, point_id: int, tensor, reqs, *, step_id: int, stream: int = 0,
                       out_dtype: Optional[int] = None, summary_mask: int = 0, keep_mask=None,
                       row_index=None, allow: Sequence[int] = ()) -> int:
        """Convenience for torch tensors on the GPU (device memory and streams only)."""
        dt = _torch_dtype_code(tensor)
        return self.observe(point_id, tensor.data_ptr(), dt, tuple(tensor.shape),
                            tuple(tensor.stride()), reqs, step_id=step_id, stream=stream,
                            out_dtype=dt if out_dtype is None else out_dtype,
                            summary_mask=summary_mask,
                            keep_mask_dev=0 if keep_mask is None else keep_mask.data_ptr(),
                            row_index_dev=0 if row_index is None else row_index.data_ptr(),
                            allow=allow)

    def observe_paged(self, point_id: int, cache, block_table, reqs, *, block_size: int,
                      n_heads: int, head_dim: int, heads_sel: Sequence[int], step_id: int,
                      stream: int = 0, out_dtype: Optional[int] = None, summary_mask: int = 0,
                      keep_mask=None, allow: Sequence[int] = ()) -> int:
        """cache: torch tensor [blocks, slots, heads, dim]; block_table: int32 [n_seqs, max_blocks]."""
        dt = _torch_dtype_code(cache)
        ra = _reqs_buffer(reqs)
        kv = PagedKV(cache.data_ptr(), dt, cache.stride(0), cache.stride(1), cache.stride(2),
                     block_size, n_heads, head_dim, cache.shape[0], block_table.shape[0],
                     block_table.data_ptr(), block_table.stride(0), len(heads_sel),
                     (C.c_uint32 * 8)(*heads_sel))
        sel = Selection(ra.shape[0], ra.ctypes.data,
                        None if keep_mask is None else keep_mask.data_ptr(), None)
        xf = Transform(dt if out_dtype is None else out_dtype, summary_mask)
        return _check(lib().dmi_observe_paged(self._h, point_id, C.byref(kv), C.byref(sel),
                                              C.byref(xf), step_id, stream or None), allow)

    def observe_batch(self, point_ids, tensors, reqs, *, step_id: int, stream: int = 0,
                      out_dtype: Optional[int] = None, summary_mask: int = 0, keep_mask=None, row_index=None,
                      paged=None, allow: Sequence[int] = ()):
        """dmi_observe_batch / dmi_observe_paged_batch (paged: an object with block_table, block_size,
        n_heads, head_dim, heads_sel; tensors are then the caches).  Returns (status, n_done)."""
        po = PreparedBatch(self, point_ids, tensors, reqs, out_dtype=out_dtype, summary_mask=summary_mask,
                           keep_mask=keep_mask, row_index=row_index, paged=paged)
        rc, done = po(step_id, stream or None)
        _check(rc, allow)
        return rc, done

    # -- consumer --------------------------------------------------------
    def drain(self, flags: int = 0, allow: Sequence[int] = ()) -> int:
        moved = C.c_uint64()
        code = _check(lib().dmi_drain(self._h, flags, C.byref(moved)), allow)
        self.last_drain_status = code
        return int(moved.value)

    def poll_host(self, max_records: int = 256) -> List[RecordView]:
        n = C.c_uint32()
        m = min(max_records, len(self._views))
        _check(lib().dmi_poll_host(self._h, self._views, m, C.byref(n)))
        return [RecordView(v.seq, v.p0 or 0, v.n0, v.p1 or 0, v.n1) for v in self._views[: n.value]]

    def poll_host_raw(self, max_records: int = 256):
        """As poll_host, without building Python objects: (n, ctypes array of views)."""
        n = C.c_uint32()
        _check(lib().dmi_poll_host(self._h, self._views, min(max_records, len(self._views)), C.byref(n)))
        return n.value, self._views

    def release_host(self, upto_seq: int):
        _check(lib().dmi_release_host(self._h, upto_seq))

    # -- policy / stats --------------------------------------------------
    def set_policy(self, mode: int, sample_k: int = 1, sample_phase: int = 0):
        p = Policy(mode, sample_k, sample_phase)
        _check(lib().dmi_set_policy(self._h, C.byref(p)))

    def point_enable(self, point_id: int, enabled: bool):
        _check(lib().dmi_point_enable(self._h, point_id, int(enabled)))

    def get_stats(self) -> Stats:
        s = StatsC()
        _check(lib().dmi_get_stats(self._h, C.byref(s)))
        return Stats(**{n: int(getattr(s, n)) for n in _STAT_FIELDS})

    def get_point_drops(self, point_id: int) -> int:
        n = C.c_uint64()
        _check(lib().dmi_get_point_drops(self._h, point_id, C.byref(n)))
        return int(n.value)

    def free_bytes(self) -> int:
        n = C.c_uint64()
        _check(lib().dmi_ring_free_bytes(self._h, C.byref(n)))
        return int(n.value)

    def set_keep_mask(self, keep, stream: int = 0) -> int:
        """Upload a keep vector; returns the device address to pass as keep_mask_dev."""
        k = np.ascontiguousarray(np.asarray(keep, dtype=np.uint8))
        out = C.c_void_p()
        _check(lib().dmi_set_keep_mask(self._h, k.ctypes.data if k.size else None, k.size, stream or None,
                                       C.byref(out)))
        return int(out.value or 0)

    # -- exporter stages 2-3 -----------------------------------------------
    def exporter_start(self, max_pageable_bytes: int, n_copy_threads: int = 0):
        _check(lib().dmi_exporter_start(self._h, max_pageable_bytes, n_copy_threads))

    def exporter_next(self, timeout_ms: int = 100) -> Optional["SliceC"]:
        """The next per-request slice, or None after timeout_ms.  Release it when done."""
        sl = SliceC()
        rc = _check(lib().dmi_exporter_next(self._h, C.byref(sl), timeout_ms), allow=(ERR_AGAIN,))
        return None if rc == ERR_AGAIN else sl

    def exporter_next_many(self, buf, timeout_ms: int = 100) -> int:
        """Fill a (SliceC * n) array with the slices ready now; returns how many."""
        n = C.c_uint32()
        _check(lib().dmi_exporter_next_many(self._h, buf, len(buf), C.byref(n), timeout_ms), allow=(ERR_AGAIN,))
        return int(n.value)

    def exporter_release_many(self, buf, n: int):
        _check(lib().dmi_exporter_release_many(self._h, buf, n))

    def exporter_release(self, sl: "SliceC"):
        _check(lib().dmi_exporter_release(self._h, C.byref(sl)))

    def exporter_stop(self):
        _check(lib().dmi_exporter_stop(self._h))

    def debug_fill_rings(self, value: int):
        _check(lib().dmi_debug_fill_rings(self._h, value))

    def debug_exporter_allocs(self):
        """(buffers taken from the allocator, records that reused an idle buffer) of the exporter's copy stage."""
        a, b = C.c_uint64(0), C.c_uint64(0)
        _check(lib().dmi_debug_exporter_allocs(self._h, C.byref(a), C.byref(b)))
        return a.value, b.value


# ---------------------------------------------------------------- the 8-bit KV cache (include/dmi_kv8.h)
# The structs as bytes, padding included, packed once for what stays and per call for what does not.
_PACK_KV8 = struct.Struct("=QQQQqqqqqIIIIIIQq").pack
_PACK_KV8_BATCH = struct.Struct("=IIIIQQQ").pack
_PACK_KV8_HEADS = struct.Struct("=QI4xqq").pack
_PACK_KV8_WEIGHT = struct.Struct("=Qqq").pack


def _typed(t, what, dtype, dims):
    import torch
    if t.dtype != getattr(torch, dtype) or t.dim() != dims:
        raise ValueError(f"{what} must be {dtype} with {dims} dimensions")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    return t


class KV8:
    """A paged cache in 8 bits (dmi_kv8_t) over the caller's tensors, which it keeps.

    k, v: [blocks, slots, heads, dim], torch.uint8 or torch.float8_e4m3fn, any strides that dmi_kv8.h allows (the same for both);
    k_scale, v_scale: fp32 [blocks, heads], the same strides; block_table: int32 [n_seqs, max_blocks]."""

    def __init__(self, k, v, k_scale, v_scale, block_table):
        import torch
        for t, what in ((k, "k"), (v, "v")):
            if t.dtype not in (torch.uint8, torch.float8_e4m3fn) or t.dim() != 4 or t.stride(3) != 1:
                raise ValueError(f"{what} must be uint8 or float8_e4m3fn [blocks, slots, heads, dim] with contiguous rows")
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.dtype != torch.float32 or t.dim() != 2:
                raise ValueError(f"{what} must be float32 [blocks, heads]")
        _typed(block_table, "block_table", "int32", 2)
        if k.shape != v.shape or k.stride() != v.stride() or k_scale.stride() != v_scale.stride() \
                or any(tuple(t.shape) != (k.shape[0], k.shape[2]) for t in (k_scale, v_scale)):
            raise ValueError("k and v must share shape and strides, and so must their scales, [blocks, heads]")
        self.k, self.v, self.k_scale, self.v_scale, self.block_table = k, v, k_scale, v_scale, block_table
        self.n_heads, self.head_dim, self.block_size = k.shape[2], k.shape[3], k.shape[1]
        self._raw = _PACK_KV8(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), k.stride(0), k.stride(1),
                              k.stride(2), k_scale.stride(0), k_scale.stride(1), k.shape[1], k.shape[2], k.shape[3], k.shape[0],
                              block_table.shape[0], block_table.shape[1], block_table.data_ptr(),
                              block_table.stride(0) if block_table.shape[0] > 1 else block_table.shape[1])


class KV8Batch:
    """The requests of a call (dmi_kv8_batch_t): int32 device tensors lens [n_reqs], starts [n_reqs + 1] or None (one new token
    each), rows [n_reqs] or None, and the host's bounds.  Their contents may change between calls, within the bounds."""

    def __init__(self, lens, *, max_len: int, starts=None, rows=None, total_new: Optional[int] = None, max_new: int = 1):
        n = lens.shape[0]
        for t, what, size in ((lens, "lens", n), (starts, "starts", n + 1), (rows, "rows", n)):
            if t is not None and _typed(t, what, "int32", 1).shape[0] != size:
                raise ValueError(f"{what} must have {size} entries")
        if total_new is None:
            if starts is not None:
                raise ValueError("starts without total_new")
            total_new = n
        self.lens, self.starts, self.rows = lens, starts, rows
        self.n_reqs, self.total_new, self.max_new, self.max_len = n, total_new, max_new, max_len
        self._raw = _PACK_KV8_BATCH(n, total_new, max_new, max_len, lens.data_ptr(), 0 if starts is None else starts.data_ptr(),
                                    0 if rows is None else rows.data_ptr())


def _kv8_heads(t, what, rows, heads, dim):
    shape = t.shape
    if len(shape) != 3 or shape[0] < rows or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{what} must be [{rows}, {heads}, {dim}], not {list(shape)}")
    stride = t.stride()
    if stride[2] != 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    return _PACK_KV8_HEADS(t.data_ptr(), _torch_dtype_code(t), stride[0], stride[1])


def _kv8_weight(t, what, rows, heads, positions):
    if t is None:
        return None
    _typed(t, what, "float32", 3)
    shape, stride = t.shape, t.stride()
    if shape[0] < rows or shape[1] != heads or shape[2] < positions:
        raise ValueError(f"{what} must be [{rows}, {heads}, {positions}] or longer, not {list(shape)}")
    return _PACK_KV8_WEIGHT(t.data_ptr(), stride[0], stride[1])


def kv8_append(cache: KV8, batch: KV8Batch, key, value, *, stream: int = 0) -> None:
    """dmi_kv8_append: key, value [total_new, heads, dim], bf16 / fp16 / fp32, into the cache."""
    k = _kv8_heads(key, "key", batch.total_new, cache.n_heads, cache.head_dim)
    v = _kv8_heads(value, "value", batch.total_new, cache.n_heads, cache.head_dim)
    _check(lib().dmi_kv8_append(cache._raw, batch._raw, k, v, stream or None))


def kv8_attend_workspace(cache: KV8, batch: KV8Batch, n_q_heads: int, with_weight: bool) -> int:
    """Bytes of workspace that kv8_attend takes."""
    return int(lib().dmi_kv8_attend_workspace(cache._raw, batch._raw, n_q_heads, int(with_weight)))


def _scratch(n, like, stream):
    """n bytes from torch's allocator, in the order of `stream`."""
    import torch
    # (the current stream's handle without the object around it: 0.1 us for 1.9)
    if not like.is_cuda or torch._C._cuda_getCurrentRawStream(like.get_device()) == stream:
        return torch.empty(n, dtype=torch.uint8, device=like.device)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=like.device)):
        return torch.empty(n, dtype=torch.uint8, device=like.device)


def kv8_attend(cache: KV8, batch: KV8Batch, q, out, *, scale: Optional[float] = None, lse=None, weight=None, prior=None,
               decay: float = 1.0, workspace=None, stream: int = 0) -> None:
    """dmi_kv8_attend: q, out [total_new, query heads, dim], bf16 or fp16; lse fp32 [total_new, query heads]; weight, prior fp32
    [n_seqs, heads, positions].  scale: dim ** -0.5 if not given.  workspace: uint8; without one it comes from torch's allocator."""
    n, heads = batch.total_new, q.shape[1]
    if weight is None and prior is not None:
        raise ValueError("prior without weight")
    if lse is not None and (tuple(lse.shape) != (n, heads) or not lse.is_contiguous()):
        raise ValueError(f"lse must be contiguous [{n}, {heads}]")
    if lse is not None and _torch_dtype_code(lse) != DT_FP32:
        raise ValueError("lse must be float32")
    raw_q = _kv8_heads(q, "q", n, heads, cache.head_dim)
    raw_out = _kv8_heads(out, "out", n, heads, cache.head_dim)
    rows = cache.block_table.shape[0]
    raw_weight = _kv8_weight(weight, "weight", rows, cache.n_heads, batch.max_len)
    raw_prior = _kv8_weight(prior, "prior", rows, cache.n_heads, batch.max_len)
    if workspace is None:
        need = lib().dmi_kv8_attend_workspace(cache._raw, batch._raw, heads, weight is not None)
        if need:
            workspace = _scratch(need, q, stream)
    _check(lib().dmi_kv8_attend(cache._raw, batch._raw, raw_q, heads, cache.head_dim ** -0.5 if scale is None else scale, raw_out,
                                None if lse is None else lse.data_ptr(), raw_weight, raw_prior, decay,
                                None if workspace is None else workspace.data_ptr(),
                                0 if workspace is None else workspace.numel() * workspace.element_size(), stream or None))


def kv8_evict(cache: KV8, batch: KV8Batch, weight, to: KV8, to_weight, *, keep: int, recent: int, positions, lens,
              stream: int = 0) -> None:
    """dmi_kv8_evict: weight fp32 [n_seqs, heads, positions] of the cache's tokens; what is kept goes into `to`, to_weight (the
    same layout, at least `keep` positions), positions int32 [n_reqs, heads, keep] and lens int32 [n_reqs]."""
    rows = cache.block_table.shape[0]
    raw_weight = _kv8_weight(weight, "weight", rows, cache.n_heads, batch.max_len)
    raw_to_weight = _kv8_weight(to_weight, "to_weight", rows, cache.n_heads, min(keep, batch.max_len))
    _typed(positions, "positions", "int32", 3)
    _typed(lens, "lens", "int32", 1)
    if tuple(positions.shape) != (batch.n_reqs, cache.n_heads, keep) or not positions.is_contiguous() \
            or lens.shape[0] != batch.n_reqs:
        raise ValueError(f"positions must be contiguous [{batch.n_reqs}, {cache.n_heads}, {keep}] and lens [{batch.n_reqs}]")
    _check(lib().dmi_kv8_evict(cache._raw, batch._raw, raw_weight, to._raw, raw_to_weight, keep, recent, positions.data_ptr(),
                               lens.data_ptr(), stream or None))


# ---------------------------------------------------------------- the 8-bit KV cache: long contexts (include/dmi_kv8_long.h)
_PACK_KV8_ROTARY = struct.Struct("=QQII").pack
_PACK_KV8_BOUNDS = struct.Struct("=Qqq").pack
_PACK_KV8_PREFIX = struct.Struct("=IIQQ").pack


class KV8Rotary:
    """How positions rotate rows of heads (dmi_kv8_rotary_t): freq fp32 [pairs], radians a position; positions int32 [total_new] or None
    (a token's place in the cache); pairs: neighbouring elements are a pair, not elements half of the rotated ones apart."""

    def __init__(self, freq, *, positions=None, pairs: bool = False):
        if not _typed(freq, "freq", "float32", 1).numel():
            raise ValueError("freq is empty")
        if positions is not None:
            _typed(positions, "positions", "int32", 1)
        self.freq, self.positions, self.rotary_dim, self.pairs = freq, positions, 2 * freq.shape[0], bool(pairs)
        self._raw = _PACK_KV8_ROTARY(freq.data_ptr(), 0 if positions is None else positions.data_ptr(), self.rotary_dim, int(self.pairs))


class KV8Prefix:
    """Groups of requests whose contexts begin alike (dmi_kv8_prefix_t): int32 device tensors group_starts [n_groups + 1] (requests)
    and prefix [n_groups] (tokens), of at most max_prefix.  Their contents may change between calls."""

    def __init__(self, group_starts, prefix, *, max_prefix: int):
        _typed(group_starts, "group_starts", "int32", 1)
        if _typed(prefix, "prefix", "int32", 1).shape[0] + 1 != group_starts.shape[0]:
            raise ValueError("group_starts must have one entry more than prefix")
        self.group_starts, self.prefix, self.n_groups, self.max_prefix = group_starts, prefix, prefix.shape[0], max_prefix
        self._raw = _PACK_KV8_PREFIX(self.n_groups, max_prefix, group_starts.data_ptr(), prefix.data_ptr())


def kv8_append_rotated(cache: KV8, batch: KV8Batch, key, value, rotary: KV8Rotary, *, q=None, q_out=None, stream: int = 0) -> None:
    """dmi_kv8_append_rotated: key (rotated) and value [total_new, heads, dim] into the cache; q [total_new, query heads, dim] rotated into
    q_out, which may be q.  bf16 / fp16 / fp32, all the same."""
    n, dim = batch.total_new, cache.head_dim
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if rotary.positions is not None and rotary.positions.shape[0] < n:
        raise ValueError(f"positions must have {n} entries")
    heads = 0 if q is None else q.shape[1]
    k = _kv8_heads(key, "key", n, cache.n_heads, dim)
    v = _kv8_heads(value, "value", n, cache.n_heads, dim)
    _check(lib().dmi_kv8_append_rotated(cache._raw, batch._raw, k, v, rotary._raw, None if q is None else _kv8_heads(q, "q", n, heads, dim),
                                        heads, None if q is None else _kv8_heads(q_out, "q_out", n, heads, dim), stream or None))


def _kv8_bounds(t, cache):
    import torch
    shape, stride = t.shape, t.stride()
    if t.dtype not in (torch.uint8, torch.float8_e4m3fn) or tuple(shape) != (cache.k.shape[0], cache.n_heads, 2, cache.head_dim) \
            or stride[3] != 1 or stride[2] != cache.head_dim:
        raise ValueError(f"bounds must be uint8 or float8_e4m3fn [{cache.k.shape[0]}, {cache.n_heads}, 2, {cache.head_dim}], the last two contiguous")
    return _PACK_KV8_BOUNDS(t.data_ptr(), stride[0], stride[1])


def kv8_bound(cache: KV8, batch: KV8Batch, bounds, *, stream: int = 0) -> None:
    """dmi_kv8_bound: bounds [blocks, heads, 2, dim] (the least, the largest) of the blocks that the call's new tokens reach."""
    _check(lib().dmi_kv8_bound(cache._raw, batch._raw, _kv8_bounds(bounds, cache), stream or None))


def _kv8_blocks(t, batch, cache):
    _typed(t, "blocks", "int32", 3)
    if t.shape[0] < batch.total_new or t.shape[1] != cache.n_heads or not t.is_contiguous():
        raise ValueError(f"blocks must be contiguous [{batch.total_new}, {cache.n_heads}, blocks of a token], not {list(t.shape)}")
    return t.data_ptr()


def _kv8_workspace(workspace, need, like, stream):
    """(the workspace, which the caller holds until its call has returned, its address, its bytes)."""
    if workspace is None and need:
        workspace = _scratch(need, like, stream)
    return (None, None, 0) if workspace is None else (workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size())


def kv8_select_workspace(cache: KV8, batch: KV8Batch, n_select: int) -> int:
    """Bytes of workspace that kv8_select takes."""
    return int(lib().dmi_kv8_select_workspace(cache._raw, batch._raw, n_select))


def kv8_select(cache: KV8, batch: KV8Batch, bounds, q, blocks, *, first: int = 1, recent: int = 2, workspace=None, stream: int = 0) -> None:
    """dmi_kv8_select: for each new token and head of the cache, blocks.shape[2] blocks, into blocks int32 [total_new, heads, n_select]: the
    first and the most recent ones, and those whose bounds allow q [total_new, query heads, dim] (bf16 or fp16) the largest scores."""
    n, n_select = batch.total_new, blocks.shape[-1]
    to = _kv8_blocks(blocks, batch, cache)
    raw_q, raw_bounds = _kv8_heads(q, "q", n, q.shape[1], cache.head_dim), _kv8_bounds(bounds, cache)
    need = 0 if workspace is not None else lib().dmi_kv8_select_workspace(cache._raw, batch._raw, n_select)
    held, at, size = _kv8_workspace(workspace, need, q, stream)
    _check(lib().dmi_kv8_select(cache._raw, batch._raw, raw_bounds, raw_q, q.shape[1], n_select, first, recent, to, at, size, stream or None))


def _kv8_lse(lse, n, heads):
    if lse is None:
        return None
    if tuple(lse.shape) != (n, heads) or not lse.is_contiguous():
        raise ValueError(f"lse must be contiguous [{n}, {heads}]")
    if _torch_dtype_code(lse) != DT_FP32:
        raise ValueError("lse must be float32")
    return lse.data_ptr()


def kv8_attend_blocks_workspace(cache: KV8, batch: KV8Batch, n_q_heads: int, n_select: int) -> int:
    """Bytes of workspace that kv8_attend_blocks takes."""
    return int(lib().dmi_kv8_attend_blocks_workspace(cache._raw, batch._raw, n_q_heads, n_select))


def kv8_attend_blocks(cache: KV8, batch: KV8Batch, blocks, q, out, *, scale: Optional[float] = None, lse=None, workspace=None,
                      stream: int = 0) -> None:
    """dmi_kv8_attend_blocks: attention of each new token over the blocks listed for it, int32 [total_new, heads, n_select] as kv8_select
    writes them; q, out, scale, lse and workspace as in kv8_attend."""
    n, heads, n_select = batch.total_new, q.shape[1], blocks.shape[-1]
    of = _kv8_blocks(blocks, batch, cache)
    raw_q, raw_out = _kv8_heads(q, "q", n, heads, cache.head_dim), _kv8_heads(out, "out", n, heads, cache.head_dim)
    need = 0 if workspace is not None else lib().dmi_kv8_attend_blocks_workspace(cache._raw, batch._raw, heads, n_select)
    held, at, size = _kv8_workspace(workspace, need, q, stream)
    _check(lib().dmi_kv8_attend_blocks(cache._raw, batch._raw, of, n_select, raw_q, heads, cache.head_dim ** -0.5 if scale is None else scale,
                                       raw_out, _kv8_lse(lse, n, heads), at, size, stream or None))


def kv8_attend_shared_workspace(cache: KV8, batch: KV8Batch, prefix: KV8Prefix, n_q_heads: int) -> int:
    """Bytes of workspace that kv8_attend_shared takes."""
    return int(lib().dmi_kv8_attend_shared_workspace(cache._raw, batch._raw, prefix._raw, n_q_heads))


def kv8_attend_shared(cache: KV8, batch: KV8Batch, prefix: KV8Prefix, q, out, *, scale: Optional[float] = None, lse=None, workspace=None,
                      stream: int = 0) -> None:
    """dmi_kv8_attend_shared: kv8_attend, without weights, of requests in groups that share the beginning of their contexts."""
    n, heads = batch.total_new, q.shape[1]
    raw_q, raw_out = _kv8_heads(q, "q", n, heads, cache.head_dim), _kv8_heads(out, "out", n, heads, cache.head_dim)
    need = 0 if workspace is not None else lib().dmi_kv8_attend_shared_workspace(cache._raw, batch._raw, prefix._raw, heads)
    held, at, size = _kv8_workspace(workspace, need, q, stream)
    _check(lib().dmi_kv8_attend_shared(cache._raw, batch._raw, prefix._raw, raw_q, heads, cache.head_dim ** -0.5 if scale is None else scale,
                                       raw_out, _kv8_lse(lse, n, heads), at, size, stream or None))
