"""ctypes binding of libgraphattn.so (argument marshalling only).

Every step of the computation runs in the HIP library; this module only turns numpy index arrays
and torch device tensors into the C ABI's structs and pointers.  If the library is not built, or
the process has no GPU, the compute entry points raise instead of falling back to anything.

Tensors are contiguous and on one device.  The calls that take a pool check the element types of the pool,
of the rows beside it and of slot words, lse and masses, and that each holds what the call reads or writes
(about a microsecond a call); ValueError otherwise.  Without a stream a call goes to the current stream of
the current device, and a pool (or mass) of another device is refused; the calls between two attention calls
refuse tensors of two devices.  Outputs that a call makes itself are made on the stream that it goes to: a program
that uses them on another one orders that, and says so to the allocator (record_stream), as for any tensor.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
from typing import Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libgraphattn.so")

GA_OK, GA_EINVAL, GA_ERANGE, GA_ENOMEM, GA_EHIP, GA_EUNSUPPORTED = 0, -1, -2, -3, -4, -5
GA_F32, GA_BF16, GA_MXFP4 = 0, 1, 2
DTYPES = {"f32": GA_F32, "bf16": GA_BF16, "mxfp4": GA_MXFP4}
STATUS_NAMES = {0: "GA_OK", -1: "GA_EINVAL", -2: "GA_ERANGE", -3: "GA_ENOMEM", -4: "GA_EHIP",
                -5: "GA_EUNSUPPORTED"}


class GraphAttnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status
        self.message = message


class SegmentTable(ctypes.Structure):
    _fields_ = [("num_segments", ctypes.c_int32),
                ("seg_len", ctypes.POINTER(ctypes.c_int32)),
                ("seg_page_offsets", ctypes.POINTER(ctypes.c_int64)),
                ("seg_pages", ctypes.POINTER(ctypes.c_int32))]


class BranchPaths(ctypes.Structure):
    _fields_ = [("num_branches", ctypes.c_int32),
                ("path_offsets", ctypes.POINTER(ctypes.c_int64)),
                ("path_segs", ctypes.POINTER(ctypes.c_int32))]


class Params(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("out_f32", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("num_segments", ctypes.c_int32), ("num_branches", ctypes.c_int32),
                ("num_entries", ctypes.c_int32), ("chunk_pages", ctypes.c_int32),
                ("rows_per_block", ctypes.c_int32), ("num_items", ctypes.c_int64),
                ("num_partial_rows", ctypes.c_int64), ("num_chains", ctypes.c_int32),
                ("num_query_rows", ctypes.c_int32), ("workgroups_per_cu", ctypes.c_int32),
                ("work_streams", ctypes.c_int32)]


class StateForest(ctypes.Structure):
    _fields_ = [("num_states", ctypes.c_int32), ("parent", ctypes.POINTER(ctypes.c_int32))]


class Advantages(ctypes.Structure):
    _fields_ = [("score", ctypes.c_void_p), ("step_reward", ctypes.c_void_p),
                ("a_cor", ctypes.c_void_p), ("a_eff", ctypes.c_void_p), ("a_dual", ctypes.c_void_p)]


class DeviceGraphC(ctypes.Structure):
    _fields_ = [("num_segments", ctypes.c_int32), ("num_branches", ctypes.c_int32),
                ("num_table_pages", ctypes.c_int64), ("num_path_segs", ctypes.c_int64),
                ("num_pages", ctypes.c_int64), ("seg_len", ctypes.c_void_p),
                ("seg_page_offsets", ctypes.c_void_p), ("seg_pages", ctypes.c_void_p),
                ("path_offsets", ctypes.c_void_p), ("path_segs", ctypes.c_void_p)]


class QKTransformC(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("norm_eps", ctypes.c_float), ("rotary_scale", ctypes.c_float),
                ("inv_freq", ctypes.c_void_p), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p)]


class LogitRulesC(ctypes.Structure):
    _fields_ = [("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
                ("presence", ctypes.c_void_p), ("temperature", ctypes.c_void_p),
                ("prompt_segments", ctypes.c_int32), ("bias_offsets", ctypes.c_void_p),
                ("bias_tokens", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
                ("num_bias", ctypes.c_int64), ("masks", ctypes.c_void_p),
                ("num_masks", ctypes.c_int32), ("mask_words", ctypes.c_int64),
                ("row_mask", ctypes.c_void_p)]


class Profile(ctypes.Structure):
    _fields_ = [("schedules", ctypes.c_int32), ("runs", ctypes.c_int32),
                ("sched_ms", ctypes.c_double), ("attn_ms", ctypes.c_double),
                ("merge_ms", ctypes.c_double)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           f"`python -m paper_2606_18954_amd.build_lib` (there is no fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    P = ctypes.POINTER
    lib.graphattn_decode.argtypes = [vp, vp, P(SegmentTable), P(BranchPaths), vp, vp, P(Params), vp]
    lib.graphattn_decode.restype = ctypes.c_int
    lib.graphattn_decode_static.argtypes = lib.graphattn_decode.argtypes
    lib.graphattn_decode_static.restype = ctypes.c_int
    lib.graphattn_plan_create.argtypes = [P(SegmentTable), P(BranchPaths), P(Params), vp, P(vp)]
    lib.graphattn_plan_create.restype = ctypes.c_int
    lib.graphattn_extend.argtypes = [vp, vp, P(SegmentTable), P(BranchPaths), P(i32), vp, vp,
                                     P(Params), vp]
    lib.graphattn_extend.restype = ctypes.c_int
    lib.graphattn_plan_create_extend.argtypes = [P(SegmentTable), P(BranchPaths), P(i32),
                                                 P(Params), vp, P(vp)]
    lib.graphattn_plan_create_extend.restype = ctypes.c_int
    lib.graphattn_kv_append.argtypes = [vp, vp, vp, vp, i32, P(Params), vp]
    lib.graphattn_kv_append.restype = ctypes.c_int
    lib.graphattn_kv_copy.argtypes = [vp, vp, vp, i32, P(Params), vp]
    lib.graphattn_kv_copy.restype = ctypes.c_int
    lib.graphattn_kv_read.argtypes = [vp, vp, i32, vp, vp, P(Params), vp]
    lib.graphattn_kv_read.restype = ctypes.c_int
    lib.graphattn_kv_page_bytes.argtypes = [P(Params)]
    lib.graphattn_kv_page_bytes.restype = i64
    lib.graphattn_page_table.argtypes = [vp, i32, i32, vp, vp, i32, i64, vp, i64, vp, vp, i64, vp]
    lib.graphattn_page_table.restype = ctypes.c_int
    lib.graphattn_slot_map.argtypes = [P(DeviceGraphC), vp, vp, vp, vp, vp, i32, vp]
    lib.graphattn_slot_map.restype = ctypes.c_int
    lib.graphattn_qkv_append.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp, i32, vp,
                                         P(QKTransformC), P(Params), vp]
    lib.graphattn_qkv_append.restype = ctypes.c_int
    lib.graphattn_process_logits.argtypes = [vp, i64, i32, i32, i32, P(LogitRulesC), P(DeviceGraphC),
                                             vp, vp, vp, vp, i64, i32, vp]
    lib.graphattn_process_logits.restype = ctypes.c_int
    lib.graphattn_equivalence_classes.argtypes = [vp, i32, i32, P(StateForest), ctypes.c_float,
                                                  vp, vp]
    lib.graphattn_equivalence_classes.restype = ctypes.c_int
    lib.graphattn_graph_suffix.argtypes = [vp, P(StateForest), vp, vp, i64, P(i64), vp]
    lib.graphattn_graph_suffix.restype = ctypes.c_int
    lib.graphattn_forest_create.argtypes = [P(StateForest), vp, P(vp)]
    lib.graphattn_forest_create.restype = ctypes.c_int
    lib.graphattn_forest_classes.argtypes = [vp, vp, i32, i32, ctypes.c_float, vp, vp, vp]
    lib.graphattn_forest_advantages.argtypes = [vp, vp, vp, vp, ctypes.c_double, ctypes.c_double,
                                                P(Advantages), vp]
    lib.graphattn_forest_advantages.restype = ctypes.c_int
    lib.graphattn_forest_classes.restype = ctypes.c_int
    lib.graphattn_forest_suffix.argtypes = [vp, vp, vp, vp, i64, P(i64), vp]
    lib.graphattn_forest_suffix.restype = ctypes.c_int
    lib.graphattn_forest_destroy.argtypes = [vp]
    lib.graphattn_forest_destroy.restype = None
    lib.graphattn_schedule.argtypes = [vp, vp]
    lib.graphattn_schedule.restype = ctypes.c_int
    lib.graphattn_plan_set_lengths.argtypes = [vp, P(i32), vp]
    lib.graphattn_plan_set_lengths.restype = ctypes.c_int
    lib.graphattn_run.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.graphattn_run.restype = ctypes.c_int
    lib.graphattn_run_mass.argtypes = [vp, vp, vp, vp, vp, ctypes.c_float, vp, vp]
    lib.graphattn_run_mass.restype = ctypes.c_int
    lib.graphattn_evict_create.argtypes = [P(SegmentTable), P(i32), i32, i32, i64, vp, P(vp)]
    lib.graphattn_evict_create.restype = ctypes.c_int
    lib.graphattn_evict_select.argtypes = [vp, vp, vp, vp, vp]
    lib.graphattn_evict_select.restype = ctypes.c_int
    lib.graphattn_evict_destroy.argtypes = [vp]
    lib.graphattn_evict_destroy.restype = None
    lib.graphattn_plan_info.argtypes = [vp, P(PlanInfo)]
    lib.graphattn_plan_info.restype = ctypes.c_int
    lib.graphattn_plan_debug_dump.argtypes = [vp, vp, P(i64), P(i32), P(i32), P(i32), P(i32),
                                              P(i64), P(i32)]
    lib.graphattn_plan_debug_dump.restype = ctypes.c_int
    lib.graphattn_plan_profile.argtypes = [vp, i32]
    lib.graphattn_plan_profile.restype = ctypes.c_int
    lib.graphattn_plan_profile_read.argtypes = [vp, P(Profile)]
    lib.graphattn_plan_profile_read.restype = ctypes.c_int
    lib.graphattn_plan_destroy.argtypes = [vp]
    lib.graphattn_plan_destroy.restype = None
    lib.graphattn_last_error.argtypes = []
    lib.graphattn_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int):
    if status != GA_OK:
        msg = load_library().graphattn_last_error().decode(errors="replace")
        raise GraphAttnError(status, msg)


def _ptr(a: np.ndarray, ctype):
    return a.ctypes.data_as(ctypes.POINTER(ctype))


class HostGraph:
    """The rollout graph's index arrays as the C structs (keeps the numpy arrays alive)."""

    def __init__(self, seg_len, seg_page_offsets, seg_pages, path_offsets, path_segs):
        self.seg_len = np.ascontiguousarray(seg_len, dtype=np.int32)
        self.seg_page_offsets = np.ascontiguousarray(seg_page_offsets, dtype=np.int64)
        self.seg_pages = np.ascontiguousarray(seg_pages, dtype=np.int32)
        self.path_offsets = np.ascontiguousarray(path_offsets, dtype=np.int64)
        self.path_segs = np.ascontiguousarray(path_segs, dtype=np.int32)
        self.st = SegmentTable(len(self.seg_len), _ptr(self.seg_len, ctypes.c_int32),
                               _ptr(self.seg_page_offsets, ctypes.c_int64),
                               _ptr(self.seg_pages, ctypes.c_int32))
        self.bp = BranchPaths(len(self.path_offsets) - 1, _ptr(self.path_offsets, ctypes.c_int64),
                              _ptr(self.path_segs, ctypes.c_int32))

    @classmethod
    def from_graph(cls, g) -> "HostGraph":
        return cls(g.seg_len, g.seg_page_offsets, g.seg_pages, g.path_offsets, g.path_segs)


def make_params(num_q_heads: int, num_kv_heads: int, head_dim: int, num_pages: int, dtype: str,
                softmax_scale: float = 0.0, out_f32: bool = False) -> Params:
    """dtype: of the pool, "f32", "bf16" or "mxfp4"."""
    if dtype not in DTYPES:
        raise ValueError(f"dtype {dtype!r} is none of {', '.join(DTYPES)}")
    return Params(num_q_heads, num_kv_heads, head_dim, 16, num_pages,
                  DTYPES[dtype], softmax_scale, int(bool(out_f32)))


_torch = None
_raw_stream = None


def _load_torch():
    """torch, and its raw getter of a device's current stream, where it has one: a Stream object costs 2.7 us, a
    third of a call that launches one small kernel; the getter 0.1 us."""
    global _torch, _raw_stream
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _torch = torch
    return torch


def _stream_handle(stream, t=None) -> int:
    """The stream's handle.  Without a stream a call goes to the current device's, where tensor t must live."""
    if stream is not None:
        return int(stream.cuda_stream)
    torch = _torch or _load_torch()
    device = torch.cuda.current_device()
    if t is not None and t.get_device() != device:
        raise ValueError(f"tensors live on device {t.get_device()}, the current one is {device}")
    if _raw_stream is None:
        return int(torch.cuda.current_stream().cuda_stream)
    return int(_raw_stream(device))


def _on(stream):
    """Where a call makes its own outputs: on its stream.  On another one a fill could run after the call, and memory
    could be taken that earlier work there still uses."""
    if stream is None:
        return contextlib.nullcontext()
    torch = _torch or _load_torch()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream.cuda_stream))
    return torch.cuda.stream(stream)


def _elsewhere(at: int, device):
    """Refuses a tensor of device `at` (-1: the host) beside others of `device`.  (Callers look first: a call of one small
    kernel costs ten microseconds, and has up to ten tensors.)"""
    if at < 0:
        raise ValueError("tensors passed to the library must live on the GPU")
    raise ValueError(f"tensors of one call live on one device, not on {device} and {at}")


def _dev_ptr(t, device=None) -> int:
    if t is None:
        return 0
    at = t.get_device()
    if at < 0 or (device is not None and at != device):
        _elsewhere(at, device)
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return int(t.data_ptr())


_LAYOUTS = None


def _layouts() -> dict:
    """By type: a pool's element type, its values per page, kv-head and channel, the type of q, K and V rows and
    its name, and what a message calls the pool."""
    global _LAYOUTS
    torch = _torch or _load_torch()
    pages = "tensor [num_pages, Hkv, 2, 16, D]"
    _LAYOUTS = {GA_F32: (torch.float32, 32, torch.float32, "f32", "an f32 pool is a float32 " + pages),
                GA_BF16: (torch.bfloat16, 32, torch.bfloat16, "bf16", "a bf16 pool is a bfloat16 " + pages),
                GA_MXFP4: (torch.uint8, 17, torch.bfloat16, "bf16",
                           "an MXFP4 pool is a uint8 tensor [num_pages, Hkv, 17 D]")}
    return _LAYOUTS


def _layout(params: Params, n: int):
    """(element type, values, type of the rows, its name, description) of the pool of a call with n rows or
    tokens; None where there is nothing to check."""
    known = (_LAYOUTS or _layouts()).get(params.dtype)
    if known is None or n == 0:                      # (refused by the library; nothing is read or written)
        return None
    element, values, row, name, what = known
    return element, values * params.head_dim * params.num_kv_heads * params.num_pages, row, name, what


def _row_sizes(params: Params, rows: int) -> tuple:
    """(values of q and out, values of lse, whether out is float32) of an attention call."""
    n = rows * params.num_q_heads
    return n * params.head_dim, n, bool(params.out_f32)


def _enter(stream, pool, layout, *rows) -> int:
    """Handle of a call's stream, once its pool and the q, K and V rows beside it are what its params say:
    tensors of another layout would be read, or written, past their end."""
    if pool is None or layout is None:               # (no pool: refused by the library)
        return _stream_handle(stream, pool) if pool is not None and pool.is_cuda else _stream_handle(stream)
    # (a tensor of the host is refused where its pointer is taken)
    handle = _stream_handle(stream, pool) if pool.is_cuda else 0
    element, values, row, name, what = layout
    if pool.dtype != element or pool.numel() < values:
        raise ValueError(what)
    for t in rows:
        if t is not None and t.dtype != row:
            raise ValueError(f"q, K and V rows beside this pool are {name}; {what}")
    return handle


def _check_rows(sizes: tuple, q, out, lse):
    """q, out and lse of an attention call."""
    values, n, wide = sizes
    if q is not None and q.numel() < values:
        raise ValueError("one row [Hq, D] of q per query")
    if out is not None:
        if out.dtype != (_torch.float32 if wide or q is None else q.dtype):
            raise ValueError("out must be float32 with out_f32, else of q's type")
        if out.numel() < values:
            raise ValueError("one row [Hq, D] of out per query")
    if lse is not None and (lse.dtype != _torch.float32 or lse.numel() < n):
        raise ValueError("lse must be float32, one row [Hq] per query")


def _check_words(*words):
    for t in words:
        if t.dtype != _torch.int32:
            raise ValueError("slot words must be int32")


def decode(q, pool, graph: HostGraph, params: Params, out=None, lse=None, stream=None):
    """graphattn_decode on torch tensors: returns (out [B, Hq, D], lse [B, Hq] float32)."""
    import torch
    lib = load_library()
    B = graph.bp.num_branches
    if out is None:
        odt = torch.float32 if params.out_f32 else q.dtype
        with _on(stream):
            out = torch.empty((B, params.num_q_heads, params.head_dim), dtype=odt, device=q.device)
    if lse is None:
        with _on(stream):
            lse = torch.empty((B, params.num_q_heads), dtype=torch.float32, device=q.device)
    handle = _enter(stream, pool, _layout(params, B), q)
    _check_rows(_row_sizes(params, B), q, out, lse)
    _check(lib.graphattn_decode(_dev_ptr(q), _dev_ptr(pool), ctypes.byref(graph.st),
                                ctypes.byref(graph.bp), _dev_ptr(out), _dev_ptr(lse),
                                ctypes.byref(params), handle))
    return out, lse


def decode_static(q, pool, graph: HostGraph, params: Params, out, lse, stream=None):
    """graphattn_decode_static: graphattn_decode with its workspace in the library's static
    device array (no allocation; the caller passes out and lse)."""
    lib = load_library()
    handle = _enter(stream, pool, _layout(params, graph.bp.num_branches), q)
    _check_rows(_row_sizes(params, graph.bp.num_branches), q, out, lse)
    _check(lib.graphattn_decode_static(_dev_ptr(q), _dev_ptr(pool), ctypes.byref(graph.st),
                                       ctypes.byref(graph.bp), _dev_ptr(out), _dev_ptr(lse),
                                       ctypes.byref(params), handle))
    return out, lse


def _counts(query_counts) -> np.ndarray:
    return np.ascontiguousarray(query_counts, dtype=np.int32)


def extend(q, pool, graph: HostGraph, query_counts, params: Params, out=None, lse=None,
           stream=None):
    """graphattn_extend on torch tensors: q [R, Hq, D] with R = sum(query_counts); returns
    (out [R, Hq, D], lse [R, Hq] float32)."""
    import torch
    lib = load_library()
    cnt = _counts(query_counts)
    if len(cnt) != graph.bp.num_branches:
        raise ValueError("one query count per branch")
    R = int(cnt.sum())
    if out is None:
        odt = torch.float32 if params.out_f32 else q.dtype
        with _on(stream):
            out = torch.empty((R, params.num_q_heads, params.head_dim), dtype=odt, device=q.device)
    if lse is None:
        with _on(stream):
            lse = torch.empty((R, params.num_q_heads), dtype=torch.float32, device=q.device)
    handle = _enter(stream, pool, _layout(params, R), q)
    _check_rows(_row_sizes(params, R), q, out, lse)
    _check(lib.graphattn_extend(_dev_ptr(q), _dev_ptr(pool), ctypes.byref(graph.st),
                                ctypes.byref(graph.bp), _ptr(cnt, ctypes.c_int32), _dev_ptr(out),
                                _dev_ptr(lse), ctypes.byref(params), handle))
    return out, lse


def kv_append(pool, k_new, v_new, slot_words, params: Params, stream=None):
    """graphattn_kv_append: k_new / v_new [n, Hkv, D], slot_words int32 [n] (device)."""
    lib = load_library()
    n = int(slot_words.numel())
    if k_new.shape[0] != n or v_new.shape[0] != n:
        raise ValueError("one K row and one V row per slot word")
    handle = _enter(stream, pool, _layout(params, n), k_new, v_new)
    _check_words(slot_words)
    size = n * params.num_kv_heads * params.head_dim
    if k_new.numel() < size or v_new.numel() < size:
        raise ValueError("K and V rows are [Hkv, D]")
    _check(lib.graphattn_kv_append(_dev_ptr(pool), _dev_ptr(k_new), _dev_ptr(v_new),
                                   _dev_ptr(slot_words), n, ctypes.byref(params), handle))


def kv_copy(pool, src_words, dst_words, params: Params, stream=None):
    """graphattn_kv_copy: src_words / dst_words int32 [n] (device)."""
    lib = load_library()
    n = int(dst_words.numel())
    if src_words.numel() != n:
        raise ValueError("one source word per destination word")
    handle = _enter(stream, pool, _layout(params, n))
    _check_words(src_words, dst_words)
    _check(lib.graphattn_kv_copy(_dev_ptr(pool), _dev_ptr(src_words), _dev_ptr(dst_words), n,
                                 ctypes.byref(params), handle))


def kv_read(pool, slot_words, params: Params, k_out=None, v_out=None, stream=None):
    """graphattn_kv_read: the K and V of the tokens at slot_words, (k [n, Hkv, D], v [n, Hkv, D]);
    rows of words outside the pool are left as they were (zero where this call allocates)."""
    torch = _torch or _load_torch()
    lib = load_library()
    n = int(slot_words.numel())
    shape = (n, params.num_kv_heads, params.head_dim)
    dt = torch.float32 if params.dtype == GA_F32 else torch.bfloat16
    if k_out is None:
        with _on(stream):
            k_out = torch.zeros(shape, dtype=dt, device=pool.device)
    if v_out is None:
        with _on(stream):
            v_out = torch.zeros(shape, dtype=dt, device=pool.device)
    if k_out.shape != shape or v_out.shape != shape:
        raise ValueError("one K row and one V row [Hkv, D] per slot word")
    if k_out.dtype != dt or v_out.dtype != dt or slot_words.dtype != torch.int32:
        raise ValueError(f"k_out and v_out must be {dt}, slot_words int32")
    handle = _enter(stream, pool, _layout(params, n))
    _check(lib.graphattn_kv_read(_dev_ptr(pool), _dev_ptr(slot_words), n, _dev_ptr(k_out),
                                 _dev_ptr(v_out), ctypes.byref(params), handle))
    return k_out, v_out


def kv_page_bytes(params: Params) -> int:
    """graphattn_kv_page_bytes: bytes of one page of the pool, all kv-heads."""
    n = int(load_library().graphattn_kv_page_bytes(ctypes.byref(params)))
    if n < 0:
        _check(n)
    return n


def empty_pool(params: Params, device="cuda"):
    """An uninitialised pool for these parameters: [num_pages, Hkv, 2, 16, D], or for MXFP4 pages
    uint8 [num_pages, Hkv, 17 D]."""
    import torch
    kv_page_bytes(params)
    n, h, d = params.num_pages, params.num_kv_heads, params.head_dim
    if params.dtype == GA_MXFP4:
        return torch.empty((n, h, 17 * d), dtype=torch.uint8, device=device)
    dt = torch.float32 if params.dtype == GA_F32 else torch.bfloat16
    return torch.empty((n, h, 2, 16, d), dtype=dt, device=device)


def _device(tensors):
    """The device of the first of some tensors that may be None; None where all are."""
    return next((t.get_device() for t in tensors if t is not None), None)


def _array(t, dtype, n: int, what: str, device=None) -> int:
    """Pointer of a contiguous tensor of this type, on this device, with n elements at least (0 for None); `what` says
    so."""
    if t is None:
        return 0
    if t.dtype != dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError(what)
    at = t.get_device()
    if at < 0 or (device is not None and at != device):
        _elsewhere(at, device)
    return t.data_ptr()


class DeviceGraph:
    """ga_device_graph: a rollout graph's index arrays as torch tensors on the device (kept, not copied: what a
    call reads is what they hold when it runs).  seg_len int32 [S], seg_page_offsets int64 [S + 1], seg_pages
    int32, path_offsets int64 [B + 1], path_segs int32; num_pages: of the pool."""

    device = None                                      # of its tensors

    def __init__(self, seg_len, seg_page_offsets, seg_pages, path_offsets, path_segs, num_pages: int):
        torch = _torch or _load_torch()
        self.tensors = (seg_len, seg_page_offsets, seg_pages, path_offsets, path_segs)
        self.num_segments, self.num_branches = int(seg_len.numel()), int(path_offsets.numel()) - 1
        self.num_pages = int(num_pages)
        if self.num_branches < 0:
            raise ValueError("path_offsets must be int64 [branches + 1]")
        S = self.num_segments
        d = self.device = seg_len.get_device()
        self.c = DeviceGraphC(
            S, self.num_branches, int(seg_pages.numel()), int(path_segs.numel()), self.num_pages,
            _array(seg_len, torch.int32, S, "seg_len must be int32, contiguous", d),
            _array(seg_page_offsets, torch.int64, S + 1, "seg_page_offsets must be int64 [segments + 1], contiguous", d),
            _array(seg_pages, torch.int32, 0, "seg_pages must be int32, contiguous", d),
            _array(path_offsets, torch.int64, 1, "path_offsets must be int64 [branches + 1], contiguous", d),
            _array(path_segs, torch.int32, 0, "path_segs must be int32, contiguous", d))
        self.ref = ctypes.byref(self.c)

    @classmethod
    def from_graph(cls, g: HostGraph, num_pages: int, device="cuda") -> "DeviceGraph":
        """A copy of a host graph's arrays on the device."""
        torch = _torch or _load_torch()
        return cls(*(torch.from_numpy(a).to(device) for a in (g.seg_len, g.seg_page_offsets, g.seg_pages,
                                                              g.path_offsets, g.path_segs)), num_pages)


def page_table(seg_len, free_pages, spare: int = 0, old_offsets=None, old_pages=None, offsets=None, pages=None,
               stream=None):
    """graphattn_page_table: (seg_page_offsets int64 [S + 1], seg_pages int32) on the device.  Every segment keeps its
    pages of the old table (its first len(old_offsets) - 1 segments) and gets more from the front of free_pages, for
    seg_len + spare tokens.  Without `pages` a tensor of all old and free pages' size is made, -1 behind the table.
    The next call's old_pages are its first total = seg_page_offsets[-1] entries, and its free_pages those behind the
    total - (old total) that this one took: nothing else marks them as taken."""
    torch = _torch or _load_torch()
    lib = load_library()
    S, known = int(seg_len.numel()), 0 if old_offsets is None else int(old_offsets.numel()) - 1
    had = 0 if old_pages is None else int(old_pages.numel())
    if known < 0 or (known > 0) > (old_pages is not None):
        raise ValueError("old_offsets [segments + 1] and old_pages come together")
    handle, d = _stream_handle(stream, seg_len) if seg_len.is_cuda else 0, seg_len.get_device()
    if offsets is None:
        with _on(stream):
            offsets = torch.empty(S + 1, dtype=torch.int64, device=seg_len.device)
    if pages is None:
        with _on(stream):
            pages = torch.full((had + int(free_pages.numel()),), -1, dtype=torch.int32, device=seg_len.device)
    _check(lib.graphattn_page_table(
        _array(seg_len, torch.int32, S, "seg_len must be int32, contiguous"), S, int(spare),
        _array(old_offsets, torch.int64, 0, "old_offsets must be int64, contiguous", d),
        _array(old_pages, torch.int32, 0, "old_pages must be int32, contiguous", d), known, had,
        _array(free_pages, torch.int32, 0, "free_pages must be int32, contiguous", d), int(free_pages.numel()),
        _array(offsets, torch.int64, S + 1, "offsets must be int64 [segments + 1], contiguous", d),
        _array(pages, torch.int32, 0, "pages must be int32, contiguous", d), int(pages.numel()), handle))
    return offsets, pages


def slot_map(graph: DeviceGraph, counts=None, token_offsets=None, slot_words=None, positions=None, branches=None,
             capacity=None, stream=None):
    """graphattn_slot_map: (token_offsets int32 [B + 1], slot_words, positions, branches int32 [capacity]) of every
    branch's newest counts[b] tokens (one each without counts).  The rows are those of the outputs that are given, else
    `capacity`, which only a call without counts knows by itself: one a branch."""
    torch = _torch or _load_torch()
    lib = load_library()
    B, given = graph.num_branches, [t for t in (slot_words, positions, branches) if t is not None]
    device, d = graph.tensors[0].device, graph.tensors[0].get_device()
    handle = _stream_handle(stream, graph.tensors[0])
    if counts is not None and capacity is None and not given:
        raise ValueError("capacity: how many rows the counts may add up to")
    n = min(int(t.numel()) for t in given) if given else B if capacity is None else int(capacity)
    if capacity is not None and n < capacity:
        raise ValueError("slot_words, positions and branches must be int32 [capacity], contiguous")
    if not given:
        with _on(stream):
            slot_words, positions, branches = (torch.empty(n, dtype=torch.int32, device=device) for _ in range(3))
    if token_offsets is None:
        with _on(stream):
            token_offsets = torch.empty(B + 1, dtype=torch.int32, device=device)
    what = "slot_words, positions and branches must be int32 [capacity], contiguous"
    _check(lib.graphattn_slot_map(
        graph.ref, _array(counts, torch.int32, B, "counts must be int32 [branches], contiguous", d),
        _array(token_offsets, torch.int32, B + 1, "token_offsets must be int32 [branches + 1], contiguous", d),
        _array(slot_words, torch.int32, n, what, d), _array(positions, torch.int32, n, what, d),
        _array(branches, torch.int32, n, what, d), n, handle))
    return token_offsets, slot_words, positions, branches


class QKTransform:
    """ga_qk_transform: the norm of each head (q_norm, k_norm float32 [D], None: no norm) and the rotation by the
    position (inv_freq float64 [rotary_dim / 2], radians a position; empty or None: none).  Channels i and i +
    rotary_dim / 2 turn together, or 2i and 2i + 1 where interleaved; scale multiplies what turns."""

    def __init__(self, head_dim: int, inv_freq=None, interleaved: bool = False, q_norm=None, k_norm=None,
                 eps: float = 1e-6, scale: float = 1.0):
        torch = _torch or _load_torch()
        rotary = 0 if inv_freq is None else 2 * int(inv_freq.numel())
        if rotary > head_dim:
            raise ValueError(f"{rotary} rotated channels of {head_dim}")
        if not scale:
            raise ValueError("scale must not be 0")
        self.head_dim, self.tensors = int(head_dim), (inv_freq, q_norm, k_norm)
        d = self.device = _device(self.tensors)
        what = "q_norm and k_norm must be float32 [head_dim], contiguous"
        self.c = QKTransformC(rotary, int(bool(interleaved)), float(eps), float(scale),
                              _array(inv_freq, torch.float64, 0, "inv_freq must be float64, contiguous", d),
                              _array(q_norm, torch.float32, head_dim, what, d),
                              _array(k_norm, torch.float32, head_dim, what, d))
        self.ref = ctypes.byref(self.c)


def _rows(t, shape: tuple, dtype, device=None) -> tuple:
    """(pointer, values from a token's heads to the next one's) of rows [n, heads, dim]; the heads of a token lie one
    behind the other."""
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"q, K and V rows beside this pool are {dtype} [tokens, heads, {shape[2]}]")
    n, heads, dim = shape
    token, head, channel = t.stride()
    if (channel != 1 or (heads > 1 and head != dim)) and n:
        raise ValueError("the heads of a token must lie one behind the other")
    at = t.get_device()
    if at < 0 or (device is not None and at != device):
        _elsewhere(at, device)
    return t.data_ptr(), token if n > 1 else heads * dim


def qkv_append(pool, q, k, v, positions, slot_words, transform: QKTransform, params: Params, q_out=None,
               stream=None):
    """graphattn_qkv_append: q [n, Hq, D] normed and rotated into q_out (returned), k [n, Hkv, D] likewise and v into the
    pool's slots.  q, k and v may be parts of one projection's rows (strided tokens); positions and slot_words int32
    [n]: a position below 0 is padding, a word outside the pool stores nothing."""
    torch = _torch or _load_torch()
    lib = _lib or load_library()
    n, Hq, Hkv, D = positions.numel(), params.num_q_heads, params.num_kv_heads, params.head_dim
    layout = _layout(params, n)
    handle = _enter(stream, pool, layout)
    row = layout[2] if layout else q.dtype
    if transform.head_dim != D:
        raise ValueError(f"a transform of {transform.head_dim}-wide heads for {D}-wide ones")
    if q_out is None:
        with _on(stream):
            q_out = torch.zeros((n, Hq, D), dtype=row, device=q.device)
    if positions.dtype != torch.int32 or slot_words.dtype != torch.int32 or slot_words.numel() < n:
        raise ValueError("positions and slot_words must be int32, one per token")
    if q_out.dtype != row or q_out.numel() < n * Hq * D:
        raise ValueError("q_out must be [tokens, Hq, D] of q's type, contiguous")
    shape, d = (n, Hkv, D), q.get_device()
    if transform.device is not None and transform.device != d:
        raise ValueError(f"the transform's tensors live on device {transform.device}, q on {d}")
    qp, qs = _rows(q, (n, Hq, D), row)
    kp, ks = _rows(k, shape, row, d)
    vp, vs = _rows(v, shape, row, d)
    status = lib.graphattn_qkv_append(_dev_ptr(pool, d), qp, kp, vp, qs, ks, vs, _dev_ptr(positions, d),
                                      _dev_ptr(slot_words, d), n, _dev_ptr(q_out, d), transform.ref, ctypes.byref(params),
                                      handle)
    if status:
        _check(status)
    return q_out


class LogitRules:
    """ga_logit_rules: per-row penalties and temperature (float32 [rows]), biases (CSR: bias_offsets int64 [rows + 1],
    bias_tokens int32 ascending within a row, bias_values float32), grammar masks (int32 or uint32 [masks, words], a
    set bit: the token may come) with row_mask int32 [rows] (outside [0, masks): none).  None leaves a rule out; the
    first prompt_segments of a path count for the repetition penalty alone."""

    device = None                                      # of its tensors

    def __init__(self, repetition=None, frequency=None, presence=None, temperature=None, prompt_segments: int = 0,
                 bias_offsets=None, bias_tokens=None, bias_values=None, masks=None, row_mask=None):
        torch = _torch or _load_torch()
        self.tensors = (repetition, frequency, presence, temperature, bias_offsets, bias_tokens, bias_values, masks,
                        row_mask)
        d = self.device = _device(self.tensors)
        per_row = [t for t in self.tensors[:4] + (row_mask,) if t is not None]
        self.rows = min((int(t.numel()) for t in per_row), default=None)
        biases = [t is not None for t in self.tensors[4:7]]
        if any(biases) != all(biases):
            raise ValueError("bias_offsets, bias_tokens and bias_values come together")
        if (masks is None) != (row_mask is None):
            raise ValueError("masks and row_mask come together")
        nb = 0
        if bias_tokens is not None:
            nb = int(bias_tokens.numel())
            at = int(bias_offsets.numel()) - 1
            self.rows = at if self.rows is None else min(self.rows, at)
        self.vocab, (nm, words) = None, (0, 0)
        if masks is not None:
            if masks.dim() != 2 or masks.element_size() != 4 or masks.is_floating_point():
                raise ValueError("masks must be int32 or uint32 [masks, words]")
            nm, words = masks.shape
            self.vocab = 32 * words
        self.counted = any(t is not None for t in self.tensors[:3])
        what = "penalties and temperature must be float32 [rows], contiguous"
        self.c = LogitRulesC(
            *(_array(t, torch.float32, 0, what, d) for t in self.tensors[:4]), int(prompt_segments),
            _array(bias_offsets, torch.int64, 1, "bias_offsets must be int64 [rows + 1], contiguous", d),
            _array(bias_tokens, torch.int32, 0, "bias_tokens must be int32, contiguous", d),
            _array(bias_values, torch.float32, nb, "bias_values must be float32, one per token, contiguous", d), nb,
            0 if masks is None else _array(masks, masks.dtype, 0, "masks must be contiguous", d), nm, words,
            _array(row_mask, torch.int32, 0, "row_mask must be int32 [rows], contiguous", d))
        self.ref = ctypes.byref(self.c)


def process_logits(logits, rules: LogitRules, graph: Optional[DeviceGraph] = None, token_ids=None, row_branches=None,
                   row_positions=None, out=None, out_f32: bool = False, stream=None):
    """graphattn_process_logits: logits [rows, vocab] (float32 or bfloat16; rows may be strided) through the rules,
    into out (returned; `logits` itself: in place).  token_ids int32 [num_pages x 16]: the token of every slot;
    row_branches and row_positions int32 [rows] as slot_map writes them (None: row r is branch r and sees its whole
    path).  Rows of padding are left as they were (zero where this call allocates)."""
    torch = _torch or _load_torch()
    lib = load_library()
    if logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("logits must be float32 or bfloat16 [rows, vocab]")
    rows, vocab = logits.shape
    handle, d = _stream_handle(stream, logits) if logits.is_cuda else 0, logits.get_device()
    if out is None:
        with _on(stream):
            out = torch.zeros((rows, vocab), dtype=torch.float32 if out_f32 else logits.dtype, device=logits.device)
    if out.shape != logits.shape or out.dtype not in (torch.float32, logits.dtype):
        raise ValueError("out must be [rows, vocab], float32 or of the logits' type")
    if rules.rows is not None and rules.rows < rows:
        raise ValueError("the rules have fewer rows than the logits")
    if rules.vocab is not None and rules.vocab < vocab:
        raise ValueError("the masks have fewer tokens than the logits")
    if rules.counted and (graph is None or token_ids is None):
        raise ValueError("penalties need the graph and its slots' token_ids")
    if rows and vocab and (logits.stride(1) != 1 or out.stride(1) != 1):
        raise ValueError("the values of a row must lie one behind the other")
    what = "row_branches and row_positions must be int32 [rows], contiguous"
    ids = _array(token_ids, torch.int32, 16 * graph.num_pages if graph is not None else 0,
                 "token_ids must be int32, one per slot of the pool, contiguous", d)
    bw, pw = _array(row_branches, torch.int32, rows, what, d), _array(row_positions, torch.int32, rows, what, d)
    if d < 0 or d != out.get_device():
        _elsewhere(min(d, out.get_device()), d)
    for x in (rules, graph):
        if x is not None and x.device is not None and x.device != d:
            raise ValueError(f"the tensors of the rules or the graph live on device {x.device}, the logits on {d}")
    si, so = (t.stride(0) if rows > 1 else vocab for t in (logits, out))
    _check(lib.graphattn_process_logits(
        logits.data_ptr(), si, rows, vocab, GA_F32 if logits.dtype == torch.float32 else GA_BF16, rules.ref,
        graph.ref if graph is not None else None, ids, bw, pw, out.data_ptr(), so,
        int(out.dtype == torch.float32), handle))
    return out


class HostForest:
    """The states' generation predecessors as the C struct (keeps the array alive)."""

    def __init__(self, parent):
        self.parent = np.ascontiguousarray(parent, dtype=np.int32)
        self.c = StateForest(len(self.parent), _ptr(self.parent, ctypes.c_int32))


def equivalence_classes(z, forest: HostForest, kappa: float, labels=None, stream=None):
    """graphattn_equivalence_classes: z [N, dim] bf16 (device); returns labels int32 [N]."""
    import torch
    lib = load_library()
    N = forest.c.num_states
    if z.dim() != 2 or z.shape[0] != N:
        raise ValueError("one embedding row per state")
    if labels is None:
        with _on(stream):
            labels = torch.empty(N, dtype=torch.int32, device=z.device)
    _check(lib.graphattn_equivalence_classes(_dev_ptr(z), int(z.shape[1]),
                                             GA_BF16 if z.dtype == torch.bfloat16 else GA_F32,
                                             ctypes.byref(forest.c), float(kappa),
                                             _dev_ptr(labels), _stream_handle(stream)))
    return labels


def graph_suffix(labels, forest: HostForest, capacity=None, stream=None):
    """graphattn_graph_suffix: returns (offsets int64 [N + 1], states int32 [total]) on the
    device; sized by a first call when capacity is not given."""
    import torch
    lib = load_library()
    N = forest.c.num_states
    total = ctypes.c_int64(0)
    cap = int(capacity) if capacity is not None else 0
    with _on(stream):
        offs = torch.empty(N + 1, dtype=torch.int64, device=labels.device)
        states = torch.empty(max(cap, 1), dtype=torch.int32, device=labels.device)
    st = lib.graphattn_graph_suffix(_dev_ptr(labels), ctypes.byref(forest.c), _dev_ptr(offs),
                                    _dev_ptr(states), cap, ctypes.byref(total),
                                    _stream_handle(stream))
    if st == GA_ERANGE and capacity is None:
        cap = int(total.value)
        with _on(stream):
            states = torch.empty(max(cap, 1), dtype=torch.int32, device=labels.device)
        st = lib.graphattn_graph_suffix(_dev_ptr(labels), ctypes.byref(forest.c), _dev_ptr(offs),
                                        _dev_ptr(states), cap, ctypes.byref(total),
                                        _stream_handle(stream))
    _check(st)
    return offs, states[:int(total.value)]


class Forest:
    """graphattn_forest_create / classes / suffix / destroy."""

    def __init__(self, parent, stream=None):
        self.lib = load_library()
        self.host = HostForest(parent)
        h = ctypes.c_void_p()
        _check(self.lib.graphattn_forest_create(ctypes.byref(self.host.c), _stream_handle(stream),
                                                ctypes.byref(h)))
        self.handle = h

    def classes(self, z, kappa: float, labels=None, edge_sim=None, stream=None):
        """Class labels; also sim(p(v), v) into edge_sim (float32 [N]) when it is given."""
        import torch
        N = self.host.c.num_states
        if labels is None:
            with _on(stream):
                labels = torch.empty(N, dtype=torch.int32, device=z.device)
        _check(self.lib.graphattn_forest_classes(
            self.handle, _dev_ptr(z), int(z.shape[1]),
            GA_BF16 if z.dtype == torch.bfloat16 else GA_F32, float(kappa), _dev_ptr(labels),
            _dev_ptr(edge_sim), _stream_handle(stream)))
        return labels

    def advantages(self, labels, reward, edge_sim, w: float, lambda_eff: float, out=None,
                   stream=None):
        """Graph reward and dual-group advantage: dict of float64 [N] device tensors (score,
        step_reward, a_cor, a_eff, a_dual)."""
        import torch
        N = self.host.c.num_states
        if out is None:
            with _on(stream):
                out = {k: torch.empty(N, dtype=torch.float64, device=labels.device)
                       for k in ("score", "step_reward", "a_cor", "a_eff", "a_dual")}
        adv = Advantages(*[_dev_ptr(out[k]) for k in ("score", "step_reward", "a_cor", "a_eff",
                                                      "a_dual")])
        _check(self.lib.graphattn_forest_advantages(
            self.handle, _dev_ptr(labels), _dev_ptr(reward), _dev_ptr(edge_sim), float(w),
            float(lambda_eff), ctypes.byref(adv), _stream_handle(stream)))
        return out

    def suffix(self, labels, offsets, states, stream=None) -> int:
        total = ctypes.c_int64(0)
        _check(self.lib.graphattn_forest_suffix(self.handle, _dev_ptr(labels), _dev_ptr(offsets),
                                                _dev_ptr(states), int(states.numel()),
                                                ctypes.byref(total), _stream_handle(stream)))
        return int(total.value)

    def suffix_total(self, labels, offsets, stream=None) -> int:
        """Entries the graph suffix needs (a call with no output buffer)."""
        total = ctypes.c_int64(0)
        st = self.lib.graphattn_forest_suffix(self.handle, _dev_ptr(labels), _dev_ptr(offsets),
                                              None, 0, ctypes.byref(total),
                                              _stream_handle(stream))
        if st not in (GA_OK, GA_ERANGE):
            _check(st)
        return int(total.value)

    def close(self):
        if self.handle:
            self.lib.graphattn_forest_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Plan:
    """graphattn_plan_create (or _create_extend with query_counts) / schedule / run /
    destroy."""

    def __init__(self, graph: HostGraph, params: Params, stream=None, query_counts=None):
        self.lib = load_library()
        self.graph = graph
        self.params = params
        h = ctypes.c_void_p()
        if query_counts is None:
            _check(self.lib.graphattn_plan_create(ctypes.byref(graph.st), ctypes.byref(graph.bp),
                                                  ctypes.byref(params), _stream_handle(stream),
                                                  ctypes.byref(h)))
        else:
            self.query_counts = _counts(query_counts)
            _check(self.lib.graphattn_plan_create_extend(
                ctypes.byref(graph.st), ctypes.byref(graph.bp),
                _ptr(self.query_counts, ctypes.c_int32), ctypes.byref(params),
                _stream_handle(stream), ctypes.byref(h)))
        self.handle = h
        # query rows of a run
        self._keep(params, int(graph.bp.num_branches if query_counts is None else self.query_counts.sum()))

    def _keep(self, params: Params, rows: int):
        """What the plan's calls are checked against (the library has its own copy of the params)."""
        self.rows = rows
        self.layout = _layout(params, rows)
        self.sizes = _row_sizes(params, rows)

    def set_lengths(self, seg_len, stream=None):
        """New segment lengths (host int32 [num_segments]); schedule again before the next run."""
        import numpy as np
        a = np.ascontiguousarray(np.asarray(seg_len, dtype=np.int32))
        _check(self.lib.graphattn_plan_set_lengths(
            self.handle, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
            _stream_handle(stream)))

    def schedule(self, stream=None):
        """Run the GPU segment scheduler (run() also schedules a plan that has no schedule)."""
        _check(self.lib.graphattn_schedule(self.handle, _stream_handle(stream)))

    def run(self, q, pool, out, lse, stream=None):
        handle = _enter(stream, pool, self.layout, q)
        _check_rows(self.sizes, q, out, lse)
        _check(self.lib.graphattn_run(self.handle, _dev_ptr(q), _dev_ptr(pool), _dev_ptr(out),
                                      _dev_ptr(lse), handle))

    def run_mass(self, q, pool, lse, mass_out, mass_in=None, decay: float = 1.0, stream=None):
        """graphattn_run_mass: the attention weight every cached token received from these rows
        (lse as run() wrote it), added to decay x mass_in (float32 [num_pages x 16]).  A slot's mass does
        not move with its token (kv_copy), and is not cleared for a new one (kv_append): the caller does both."""
        handle = _enter(stream, pool, self.layout, q)
        if q.numel() < self.sizes[0] or lse.numel() < self.sizes[1]:
            raise ValueError("one row of q and of lse per query")
        for t in (mass_out, mass_in):
            if t is not None and t.numel() < 16 * self.params.num_pages:
                raise ValueError("one mass per slot of the pool")
        if any(t is not None and t.dtype != _torch.float32 for t in (lse, mass_out, mass_in)):
            raise ValueError("lse and the masses must be float32")
        _check(self.lib.graphattn_run_mass(self.handle, _dev_ptr(q), _dev_ptr(pool), _dev_ptr(lse),
                                           _dev_ptr(mass_in), float(decay), _dev_ptr(mass_out),
                                           handle))
        return mass_out

    def info(self) -> PlanInfo:
        inf = PlanInfo()
        _check(self.lib.graphattn_plan_info(self.handle, ctypes.byref(inf)))
        return inf

    def debug_dump(self, stream=None):
        """Device schedule as numpy arrays: group offsets/branches, entry ranks, items, chunks
        and each branch's partial-row list (CSR)."""
        inf = self.info()
        S, E, R = inf.num_segments, inf.num_entries, inf.num_query_rows
        goff = np.zeros(S + 1, dtype=np.int64)
        gbr = np.zeros(max(E, 1), dtype=np.int32)
        rk = np.zeros(max(E, 1), dtype=np.int32)
        nit = max(int(inf.num_items), 0)
        items = np.zeros(max(3 * nit, 3), dtype=np.int32)
        nch = np.zeros(max(S, 1), dtype=np.int32)
        boff = np.zeros(R + 1, dtype=np.int64)
        bpart = np.zeros(max(int(inf.num_partial_rows), 1), dtype=np.int32)
        _check(self.lib.graphattn_plan_debug_dump(
            self.handle, _stream_handle(stream), _ptr(goff, ctypes.c_int64),
            _ptr(gbr, ctypes.c_int32), _ptr(rk, ctypes.c_int32), _ptr(items, ctypes.c_int32),
            _ptr(nch, ctypes.c_int32), _ptr(boff, ctypes.c_int64), _ptr(bpart, ctypes.c_int32)))
        return {"group_offsets": goff, "group_branches": gbr[:E], "entry_ranks": rk[:E],
                "items": items[:3 * nit].reshape(nit, 3), "segment_chunks": nch[:S],
                "branch_part_offsets": boff, "branch_parts": bpart[:int(boff[-1])]}

    def profile(self, max_calls: int):
        """Record HIP-event kernel times for the next ``max_calls`` schedule/run calls."""
        _check(self.lib.graphattn_plan_profile(self.handle, int(max_calls)))

    def profile_read(self) -> Profile:
        pr = Profile()
        _check(self.lib.graphattn_plan_profile_read(self.handle, ctypes.byref(pr)))
        return pr

    def close(self):
        if self.handle:
            self.lib.graphattn_plan_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Evict:
    """graphattn_evict_create / select / destroy: the tokens of every segment that stay.

    offsets [S + 1] (host int64): where each segment's tokens start in the selection's outputs."""

    def __init__(self, graph: HostGraph, keep_counts, first: int, recent: int, num_pages: int,
                 stream=None):
        self.handle = None
        self.lib = load_library()
        keep = np.ascontiguousarray(keep_counts, dtype=np.int32)
        if len(keep) != graph.st.num_segments:
            raise ValueError("one keep count per segment")
        self.offsets = np.concatenate([[0], np.cumsum(keep, dtype=np.int64)])
        self.num_pages = int(num_pages)
        h = ctypes.c_void_p()
        _check(self.lib.graphattn_evict_create(ctypes.byref(graph.st), _ptr(keep, ctypes.c_int32),
                                               int(first), int(recent), int(num_pages),
                                               _stream_handle(stream), ctypes.byref(h)))
        self.handle = h

    @property
    def total(self) -> int:
        """Tokens that stay, over all segments."""
        return int(self.offsets[-1])

    def select(self, mass, positions=None, slot_words=None, stream=None):
        """(positions, slot_words), int32 [total] each, from the mass of every slot."""
        import torch
        if mass.numel() < 16 * self.num_pages or mass.dtype != torch.float32:
            raise ValueError("one mass per slot of the pool, float32")
        if positions is None:
            with _on(stream):
                positions = torch.empty(self.total, dtype=torch.int32, device=mass.device)
        if slot_words is None:
            with _on(stream):
                slot_words = torch.empty(self.total, dtype=torch.int32, device=mass.device)
        if positions.numel() < self.total or slot_words.numel() < self.total:
            raise ValueError("one position and one slot word per token that stays")
        if positions.dtype != torch.int32 or slot_words.dtype != torch.int32:
            raise ValueError("positions and slot_words must be int32")
        if self.total:
            _check(self.lib.graphattn_evict_select(self.handle, _dev_ptr(mass),
                                                   _dev_ptr(positions), _dev_ptr(slot_words),
                                                   _stream_handle(stream, mass)))
        return positions, slot_words

    def close(self):
        if self.handle:
            self.lib.graphattn_evict_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def validate_only(graph: HostGraph, params: Params, query_counts=None) -> int:
    """Run the library's host-side validation through graphattn_decode (graphattn_extend with
    query_counts) with NULL device buffers; used by CPU tests of the error paths.  Returns the
    status (only meaningful for invalid inputs, which are rejected before any HIP call)."""
    lib = load_library()
    if query_counts is None:
        return lib.graphattn_decode(None, None, ctypes.byref(graph.st), ctypes.byref(graph.bp),
                                    None, None, ctypes.byref(params), None)
    cnt = _counts(query_counts)
    return lib.graphattn_extend(None, None, ctypes.byref(graph.st), ctypes.byref(graph.bp),
                                _ptr(cnt, ctypes.c_int32) if len(cnt) else None, None, None,
                                ctypes.byref(params), None)


def last_error() -> str:
    return load_library().graphattn_last_error().decode(errors="replace")


def header_symbols(header: str = "graphattn.h") -> list:
    """Function names declared in include/graphattn.h (or another header there)."""
    import re
    hdr = os.path.join(os.path.dirname(_PKG), "include", header)
    text = open(hdr).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(graphattn_\w+)\s*\(", text)))
