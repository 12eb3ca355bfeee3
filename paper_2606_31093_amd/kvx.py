"""Python binding of libkvx (include/kvx.h): argument marshalling only.

Every step of the copy runs in the library's HIP kernels.  PyTorch supplies
device memory and the stream: tensors are passed as raw pointers and the
kernels run on ``torch.cuda.current_stream()`` unless a stream is given.
The functions keep the C names: ``kvx_transfer``, ``kvx_transfer_slice``,
``kvx_transfer_layered``, ``kvx_transfer_planned``,
``kvx_transfer_layered_planned``, ``kvx_gather``, ``kvx_scatter``,
``kvx_gather_slice``, ``kvx_scatter_slice`` and ``kvx_page_hashes``, and the
calls that compute with a paged cache, ``kvx_append``, ``kvx_attend``,
``kvx_select_kept`` and ``kvx_transfer_kept`` for a decode step, and
``kvx_append_normed``, ``kvx_attend_prompt``, ``kvx_attend_tree`` and
``kvx_keep_path`` for several tokens of a request.  A missing or unloadable
library raises; there is no fallback path.

Pool and buffer shapes are duck-typed: a pool shape has integer attributes
``L C H D T N e`` and a ``layout`` name; a buffer shape has ``L C H D e``
and ``cap`` (elements).  ``paper_2606_31093_amd.workloads.PoolSpec`` and
``BufSpec`` fit.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
from dataclasses import dataclass
from typing import Any

import numpy as np

from . import build_lib

LAYOUTS = {"LPCTHD": 0, "LPCHTD": 1, "PLCTHD": 2, "PLCHTD": 3}

DERR_SRC_PAGE = 1
DERR_DST_PAGE = 2
DERR_PT_RANGE = 4
DERR_BAD_REQ = 8
DERR_STALLED = 16
DERR_BAD_PLAN = 32

STATUS = {0: "KVX_OK", -1: "KVX_ERR_NULL", -2: "KVX_ERR_SHAPE", -3: "KVX_ERR_ALIGN",
          -4: "KVX_ERR_LAYOUT", -5: "KVX_ERR_RANGE", -6: "KVX_ERR_HIP"}

REQ_DTYPE = np.dtype([("src_pt_off", "<i8"), ("dst_pt_off", "<i8"), ("buf_off", "<i8"),
                      ("src_start", "<i4"), ("dst_start", "<i4"), ("n_tokens", "<i4"),
                      ("reserved", "<i4")])


REQ_DTYPE_SIZE = REQ_DTYPE.itemsize

HASH_REQ_DTYPE = np.dtype([("payload_off", "<i8"), ("out_off", "<i8"), ("seed", "<u8"),
                           ("n_positions", "<i4"), ("reserved", "<i4")])


class Pool(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("num_layers", ctypes.c_int32),
                ("num_kv", ctypes.c_int32), ("num_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("elem_bytes", ctypes.c_int32),
                ("layout", ctypes.c_int32)]


class Buf(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("num_layers", ctypes.c_int32),
                ("num_kv", ctypes.c_int32), ("num_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("elem_bytes", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("capacity_elems", ctypes.c_int64)]


class Slice(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in (
        "src_layer0", "dst_layer0", "num_layers", "src_kv0", "dst_kv0", "num_kv",
        "src_head0", "dst_head0", "num_heads", "reserved")]


def slice_desc(sl) -> Slice:
    """A kvx_slice from (src_layer0, dst_layer0, num_layers, src_kv0, dst_kv0,
    num_kv, src_head0, dst_head0, num_heads)."""
    if isinstance(sl, Slice):
        return sl
    vals = [int(x) for x in sl]
    if len(vals) != 9:
        raise ValueError("a slice has nine fields")
    return Slice(*vals, 0)


class KvxError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


_LIB = None


def library_path() -> str:
    return os.environ.get("KVX_LIBRARY", build_lib.LIBRARY)


def lib() -> ctypes.CDLL:
    """The loaded libkvx.so.  Raises if it is missing: build it with
    ``python -m paper_2606_31093_amd.build_lib`` (or ``__graft_entry__.build()``)."""
    global _LIB
    if _LIB is None:
        _LIB = load(library_path())
    return _LIB


def load(path: str) -> ctypes.CDLL:
    """Load a build of the library at ``path`` and declare its entry points'
    argument types (``lib()`` does this once for the default build)."""
    if not os.path.exists(path):
        raise RuntimeError(f"libkvx is not built ({path} missing); run "
                           "python -m paper_2606_31093_amd.build_lib")
    # PyTorch ships its own HIP runtime.  Loaded first, it is the one
    # libkvx binds to (same soname), so the library and torch share one
    # runtime: the one that owns the tensors and streams passed in.
    # Loading libkvx first would bring a second HIP and HSA runtime into
    # the process, and one of them then finds no device.
    import torch  # noqa: F401
    L = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    pp, bp = ctypes.POINTER(Pool), ctypes.POINTER(Buf)
    L.kvx_transfer.argtypes = [pp, pp, vp, i64, vp, i64, vp, i32, vp, vp]
    L.kvx_transfer_slice.argtypes = [pp, pp, ctypes.POINTER(Slice), vp, i64, vp, i64, vp, i32,
                                     vp, vp]
    L.kvx_transfer_layered.argtypes = [pp, pp, ctypes.POINTER(Slice), vp, i64, vp, i64, vp,
                                       i32, i32, ctypes.POINTER(vp), i32, vp, vp]
    L.kvx_gather.argtypes = [pp, bp, vp, i64, vp, i32, vp, vp]
    L.kvx_scatter.argtypes = [bp, pp, vp, i64, vp, i32, vp, vp]
    sp = ctypes.POINTER(Slice)
    L.kvx_gather_slice.argtypes = [pp, bp, sp, vp, i64, vp, i32, vp, vp]
    L.kvx_scatter_slice.argtypes = [bp, pp, sp, vp, i64, vp, i32, vp, vp]
    for f in (L.kvx_transfer, L.kvx_transfer_slice, L.kvx_transfer_layered, L.kvx_gather,
              L.kvx_scatter, L.kvx_gather_slice, L.kvx_scatter_slice):
        f.restype = ctypes.c_int
    L.kvx_transfer_planned.argtypes = [pp, pp, ctypes.POINTER(Slice), vp, i64, vp, i64, vp, i32,
                                       vp, i64, i64, vp, vp]
    L.kvx_transfer_planned.restype = ctypes.c_int
    L.kvx_transfer_layered_planned.argtypes = [pp, pp, ctypes.POINTER(Slice), vp, i64, vp, i64, vp,
                                               i32, i32, ctypes.POINTER(vp), i32, vp, i64, i64, vp, vp]
    L.kvx_transfer_layered_planned.restype = ctypes.c_int
    L.kvx_plan_pages.argtypes = [vp, i32, i32, i32, vp, vp]
    L.kvx_plan_pages.restype = ctypes.c_int64
    L.kvx_plan_fill.argtypes = [vp, i32, i32, i32, i64, vp]
    L.kvx_plan_fill.restype = ctypes.c_int
    L.kvx_page_hashes.argtypes = [vp, i64, i32, i32, vp, i32, vp, i64, vp, vp]
    L.kvx_page_hashes.restype = ctypes.c_int
    L.kvx_pool_bytes.argtypes = [pp]
    L.kvx_pool_bytes.restype = ctypes.c_int64
    L.kvx_strerror.argtypes = [ctypes.c_int]
    L.kvx_strerror.restype = ctypes.c_char_p
    L.kvx_last_error.argtypes = []
    L.kvx_last_error.restype = ctypes.c_char_p
    L.kvx_abi_version.argtypes = []
    L.kvx_abi_version.restype = ctypes.c_int
    L.kvx_set_launch_choice.argtypes = [ctypes.c_int]
    L.kvx_set_launch_choice.restype = ctypes.c_int
    L.kvx_launch_choice.argtypes = []
    L.kvx_launch_choice.restype = ctypes.c_int
    L.kvx_last_launch.argtypes = []
    L.kvx_last_launch.restype = ctypes.c_int
    L.kvx_append.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, i64, vp, i32, i32, vp, vp]
    L.kvx_append.restype = ctypes.c_int
    L.kvx_append_normed.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp, i32, i32, vp, vp]
    L.kvx_append_normed.restype = ctypes.c_int
    for f in (L.kvx_attend_prompt, L.kvx_attend_tree):
        f.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, i64, vp] + [vp] * (f is L.kvx_attend_tree) + [i32, i32, i32, vp, i64,
                                                                                                 vp, vp]
        f.restype = ctypes.c_int
    L.kvx_queries_workspace.argtypes = [vp, i32, i32, i32, i32, i32]
    L.kvx_queries_workspace.restype = i64
    L.kvx_keep_path.argtypes = [vp, vp, i64, vp, i32, i32, vp, i64, vp, vp]
    L.kvx_keep_path.restype = ctypes.c_int
    L.kvx_attend.argtypes = [vp, i32, vp, vp, vp, vp, ctypes.c_float, vp, i64, vp, i32, i32, vp, i64, i64, vp, i64, vp,
                             vp]
    L.kvx_attend.restype = ctypes.c_int
    L.kvx_attend_workspace.argtypes = [vp, i32, i32, i32, i32, i32]
    L.kvx_attend_workspace.restype = i64
    L.kvx_select_kept.argtypes = [vp, i64, i64, i32, vp, i32, i32, vp, i64, i64, vp, i64, i64, vp, vp]
    L.kvx_select_kept.restype = ctypes.c_int
    L.kvx_transfer_kept.argtypes = [vp, vp, vp, vp, i64, vp, i64, vp, i32, i32, vp, i64, i64, vp, vp]
    L.kvx_transfer_kept.restype = ctypes.c_int
    # The copy calls once more, with descriptors as packed bytes: a ctypes
    # structure per descriptor and call took half of a small call's time.
    for f in _PACKED:
        g = L["kvx_" + f]
        g.argtypes = [vp if t in (pp, bp, sp) else t for t in getattr(L, "kvx_" + f).argtypes]
        g.restype = ctypes.c_int
        setattr(L, "packed_" + f, g)
    return L


_PACKED = ("transfer", "transfer_slice", "transfer_layered", "transfer_planned", "transfer_layered_planned", "gather", "scatter", "gather_slice", "scatter_slice")


# ---------------------------------------------------------------------------
# descriptors
# ---------------------------------------------------------------------------

def _ptr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def pool_desc(spec, data=None) -> Pool:
    """A kvx_pool for a pool shape; ``data`` is a tensor (or raw address)."""
    return Pool(_ptr(data), spec.L, spec.C, spec.H, spec.D, spec.T, spec.N, spec.e,
                LAYOUTS[spec.layout] if isinstance(spec.layout, str) else int(spec.layout))


def buf_desc(spec, data=None) -> Buf:
    return Buf(_ptr(data), spec.L, spec.C, spec.H, spec.D, spec.e, 0, spec.cap)


def pack_reqs(rows) -> np.ndarray:
    """(n, 6) int64 rows ``src_pt_off, dst_pt_off, buf_off, src_start,
    dst_start, n_tokens`` -> kvx_req records (numpy structured array)."""
    rows = np.asarray(rows, dtype=np.int64).reshape(-1, 6)
    out = np.zeros(len(rows), dtype=REQ_DTYPE)
    for i, name in enumerate(("src_pt_off", "dst_pt_off", "buf_off")):
        out[name] = rows[:, i]
    for i, name in ((3, "src_start"), (4, "dst_start"), (5, "n_tokens")):
        col = rows[:, i]
        if ((col < -2**31) | (col >= 2**31)).any():
            raise ValueError(f"{name} does not fit int32")
        out[name] = col
    return out


def _records(rows) -> np.ndarray:
    """kvx_req records: ``rows`` itself if it already is a record array,
    else pack_reqs(rows)."""
    if isinstance(rows, np.ndarray) and rows.dtype == REQ_DTYPE:
        return rows
    return pack_reqs(rows)


def device_reqs(rows, device="cuda"):
    """kvx_req records as a device tensor (bytes)."""
    import torch
    recs = pack_reqs(rows)
    t = torch.from_numpy(recs.view(np.uint8).copy())
    return t.to(device)


def device_table(pt, device="cuda"):
    import torch
    a = np.ascontiguousarray(np.asarray(pt if pt is not None else [], dtype=np.int32))
    return torch.from_numpy(a).to(device)


def pool_bytes(spec) -> int:
    return int(lib().kvx_pool_bytes(ctypes.byref(pool_desc(spec, 0))))


# ---------------------------------------------------------------------------
# entry points
# ---------------------------------------------------------------------------

def _stream(stream) -> int | None:
    if stream is None:
        import torch
        c = torch._C
        return c._cuda_getCurrentRawStream(c._cuda_getDevice())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int) -> None:
    if status != 0:
        raise KvxError(status, lib().kvx_last_error().decode())


_POOL_PACK = struct.Struct("=Q8i").pack
_BUF_PACK = struct.Struct("=Q6iq").pack
_SLICE_PACK = struct.Struct("=10i").pack


def _n_reqs(reqs) -> int:
    n, rest = divmod(reqs.nbytes, REQ_DTYPE_SIZE)
    if rest:
        raise ValueError("reqs must hold whole 40-byte kvx_req records")
    if not reqs.is_contiguous():
        raise ValueError("reqs must be contiguous")
    return n


def _table(t, name: str):
    """A page table, a contiguous tensor of 32-bit entries (or None): its
    address and length."""
    if t is None:
        return None, 0
    if isinstance(t, int):
        raise ValueError(f"{name} must be a contiguous int32 tensor (got an address)")
    if t.element_size() != 4 or t.is_floating_point() or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor (got {t.dtype})")
    return t.data_ptr(), t.numel()


def _err_word(t):
    """The optional device error word, one 32-bit integer: its address."""
    if t is None or isinstance(t, int):
        return t
    if t.element_size() != 4 or t.is_floating_point() or t.numel() < 1:
        raise ValueError(f"dev_err must be a 32-bit integer tensor (got {t.dtype})")
    return t.data_ptr()


def _need(t, nbytes: int, name: str) -> int:
    """The address of a tensor argument, which must hold at least the bytes
    its descriptor names."""
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    have = t.nbytes
    if have < nbytes:
        raise ValueError(f"{name} holds {have} bytes, its descriptor needs {nbytes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _pool_arg(spec, t, name: str) -> bytes:
    """The kvx_pool of a pool argument, packed."""
    L, C, H, D, T, N, e = spec.L, spec.C, spec.H, spec.D, spec.T, spec.N, spec.e
    ptr = _need(t, L * C * H * D * T * N * e, name)
    layout = spec.layout
    code = LAYOUTS[layout] if isinstance(layout, str) else int(layout)
    try:
        return _POOL_PACK(ptr, L, C, H, D, T, N, e, code)
    except struct.error:               # a value of another width: as ctypes takes it
        return bytes(pool_desc(spec, t))


def _buf_arg(spec, t, name: str) -> bytes:
    """The kvx_buf of a buffer argument, packed."""
    cap, e = spec.cap, spec.e
    ptr = _need(t, cap * e, name)
    try:
        return _BUF_PACK(ptr, spec.L, spec.C, spec.H, spec.D, e, 0, cap)
    except struct.error:
        return bytes(buf_desc(spec, t))


def _slice_arg(sl) -> bytes:
    """A kvx_slice, packed."""
    if type(sl) is tuple and len(sl) == 9:
        try:
            return _SLICE_PACK(*sl, 0)
        except struct.error:
            pass
    return bytes(slice_desc(sl))


def kvx_transfer(src, src_spec, dst, dst_spec, src_pt, dst_pt, reqs, dev_err=None,
                 stream=None) -> None:
    """Pool -> pool (see kvx_transfer in include/kvx.h).  ``src_pt`` /
    ``dst_pt`` are int32 device tensors, ``reqs`` a device tensor from
    ``device_reqs``, ``dev_err`` an optional int32/uint32 device word."""
    S, D = _pool_arg(src_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    spt, n_spt = _table(src_pt, "src_pt")
    dpt, n_dpt = _table(dst_pt, "dst_pt")
    err = _err_word(dev_err)
    _check(lib().packed_transfer(S, D, spt, n_spt, dpt, n_dpt, reqs.data_ptr(), _n_reqs(reqs), err,
                                 _stream(stream)))


def kvx_transfer_slice(src, src_spec, dst, dst_spec, sl, src_pt, dst_pt, reqs, dev_err=None,
                       stream=None) -> None:
    """Slice of a pool -> slice of another pool (see kvx_transfer_slice in
    include/kvx.h).  ``sl`` is a ``Slice`` or the nine range fields."""
    S, D = _pool_arg(src_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    X = _slice_arg(sl)
    spt, n_spt = _table(src_pt, "src_pt")
    dpt, n_dpt = _table(dst_pt, "dst_pt")
    err = _err_word(dev_err)
    _check(lib().packed_transfer_slice(S, D, X, spt, n_spt, dpt, n_dpt, reqs.data_ptr(), _n_reqs(reqs), err,
                                       _stream(stream)))


def kvx_transfer_planned(src, src_spec, dst, dst_spec, src_pt, dst_pt, reqs, plan, plan_pages,
                         plan_tokens, sl=None, dev_err=None, stream=None, library=None) -> None:
    """Pool -> pool with a plan (see kvx_transfer_planned in
    include/kvx.h): ``plan`` a device tensor holding the plan, and
    ``plan_pages``, ``plan_tokens`` its totals, as ``device_plan`` returns.  ``sl`` is an optional
    slice (nine range fields or a ``Slice``); ``library`` a build loaded with
    ``load`` (default: ``lib()``)."""
    S, D = _pool_arg(src_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    X = _slice_arg(sl) if sl is not None else None
    spt, n_spt = _table(src_pt, "src_pt")
    dpt, n_dpt = _table(dst_pt, "dst_pt")
    err = _err_word(dev_err)
    n = _n_reqs(reqs)
    if plan is not None and not isinstance(plan, int):
        if not plan.is_contiguous() or plan.nbytes < plan_bytes(n, plan_pages):
            raise ValueError("plan must be a contiguous tensor of KVX_PLAN_BYTES(n_reqs, plan_pages) "
                             "bytes")
    L = library or lib()
    status = L.packed_transfer_planned(S, D, X, spt, n_spt, dpt, n_dpt, reqs.data_ptr(), n, _ptr(plan),
                                       int(plan_pages), int(plan_tokens), err, _stream(stream))
    if status != 0:
        raise KvxError(status, L.kvx_last_error().decode())


def plan_pages(rows, page_tokens: int, side: int = 1):
    """kvx_plan_pages on a host copy of the (n, 6) rows: the exclusive prefix
    of pages per record (numpy int64, n + 1 entries), the total of pages and
    the tokens of the well-formed records, for side 0 (source) or 1
    (destination) of a pool with ``page_tokens`` tokens per page.  ``rows``
    may also be a kvx_req record array."""
    recs = _records(rows)
    prefix = np.zeros(len(recs) + 1, np.int64)
    tokens = ctypes.c_int64(0)
    n = int(lib().kvx_plan_pages(recs.ctypes.data if len(recs) else None, len(recs), int(page_tokens),
                                 int(side), prefix.ctypes.data, ctypes.byref(tokens)))
    if n < 0:
        raise KvxError(-5, lib().kvx_last_error().decode())
    return prefix, n, tokens.value


def plan_bytes(n_reqs: int, plan_pages: int) -> int:
    """KVX_PLAN_BYTES: the prefix (n_reqs + 1 int64) and the 32-byte slots."""
    return (int(n_reqs) + 1) * 8 + int(plan_pages) * 32


def host_plan(rows, src_page_tokens: int, dst_page_tokens: int):
    """kvx_plan_fill for the (n, 6) rows (or a kvx_req record array): the
    plan as a host int64 array (the prefix, then four words per slot), its
    pages and its tokens."""
    recs = _records(rows)
    _, pages, tokens = plan_pages(recs, dst_page_tokens, 1)
    buf = np.zeros(plan_bytes(len(recs), pages) // 8, np.int64)
    st = lib().kvx_plan_fill(recs.ctypes.data if len(recs) else None, len(recs), int(src_page_tokens),
                             int(dst_page_tokens), pages, buf.ctypes.data)
    if st != 0:
        raise KvxError(st, lib().kvx_last_error().decode())
    return buf, pages, tokens


def plan_slots(buf, n_reqs: int):
    """The slots of a host plan as an (pages, 8) int32 array (a view):
    dst_idx, src_idx, dst_slot, n_tokens, src_slot, req and two reserved."""
    return buf[n_reqs + 1:].view(np.int32).reshape(-1, 8)


def device_plan(rows, src_page_tokens: int, dst_page_tokens: int, device="cuda"):
    """The plan of ``rows`` on the device: (tensor, pages, tokens), the
    arguments of kvx_transfer_planned after the records."""
    import torch
    buf, pages, tokens = host_plan(rows, src_page_tokens, dst_page_tokens)
    return torch.from_numpy(buf).to(device), pages, tokens


def _event_handles(events, st, stream):
    """hipEvent_t handles of ``events`` (torch.cuda.Event objects or raw
    handles) as a ctypes array, and their count."""
    import torch
    handles = []
    for ev in events:
        if isinstance(ev, int):
            handles.append(ev)
            continue
        if not ev.cuda_event:          # torch creates the HIP event on first record
            ev.record(torch.cuda.ExternalStream(st) if stream is not None else None)
        handles.append(ev.cuda_event)
    return (ctypes.c_void_p * max(1, len(handles)))(*handles), len(handles)


def kvx_transfer_layered(src, src_spec, dst, dst_spec, src_pt, dst_pt, reqs, layers_per_group,
                         events, sl=None, dev_err=None, stream=None) -> None:
    """Layer-pipelined pool -> pool (see kvx_transfer_layered in
    include/kvx.h).  ``events`` are ``torch.cuda.Event`` objects (or raw
    hipEvent_t handles), one per layer group; the library records events[g]
    on the stream once group g has been copied."""
    S, D = _pool_arg(src_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    X = None if sl is None else _slice_arg(sl)
    spt, n_spt = _table(src_pt, "src_pt")
    dpt, n_dpt = _table(dst_pt, "dst_pt")
    err = _err_word(dev_err)
    st = _stream(stream)
    arr, n_ev = _event_handles(events, st, stream)
    _check(lib().packed_transfer_layered(S, D, X, spt, n_spt, dpt, n_dpt, reqs.data_ptr(), _n_reqs(reqs),
                                         int(layers_per_group), arr, n_ev, err, st))


def kvx_transfer_layered_planned(src, src_spec, dst, dst_spec, src_pt, dst_pt, reqs, layers_per_group,
                                 events, plan, plan_pages, plan_tokens, sl=None, dev_err=None,
                                 stream=None, library=None) -> None:
    """kvx_transfer_layered with a plan (see kvx_transfer_layered_planned
    in include/kvx.h); the plan as ``device_plan`` returns it."""
    S, D = _pool_arg(src_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    X = None if sl is None else _slice_arg(sl)
    spt, n_spt = _table(src_pt, "src_pt")
    dpt, n_dpt = _table(dst_pt, "dst_pt")
    err = _err_word(dev_err)
    n = _n_reqs(reqs)
    if plan is not None and not isinstance(plan, int):
        if not plan.is_contiguous() or plan.nbytes < plan_bytes(n, plan_pages):
            raise ValueError("plan must be a contiguous tensor of KVX_PLAN_BYTES(n_reqs, plan_pages) "
                             "bytes")
    st = _stream(stream)
    arr, n_ev = _event_handles(events, st, stream)
    L = library or lib()
    status = L.packed_transfer_layered_planned(S, D, X, spt, n_spt, dpt, n_dpt, reqs.data_ptr(), n,
                                               int(layers_per_group), arr, n_ev, _ptr(plan), int(plan_pages),
                                               int(plan_tokens), err, st)
    if status != 0:
        raise KvxError(status, L.kvx_last_error().decode())


def kvx_gather(src, src_spec, dst, buf_spec, src_pt, reqs, dev_err=None, stream=None) -> None:
    """Pool -> flat buffer (see kvx_gather in include/kvx.h)."""
    S, B = _pool_arg(src_spec, src, "src"), _buf_arg(buf_spec, dst, "dst")
    pt, n_pt = _table(src_pt, "src_pt")
    err = _err_word(dev_err)
    _check(lib().packed_gather(S, B, pt, n_pt, reqs.data_ptr(), _n_reqs(reqs), err, _stream(stream)))


def kvx_scatter(src, buf_spec, dst, dst_spec, dst_pt, reqs, dev_err=None, stream=None) -> None:
    """Flat buffer -> pool (see kvx_scatter in include/kvx.h)."""
    B, D = _buf_arg(buf_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    pt, n_pt = _table(dst_pt, "dst_pt")
    err = _err_word(dev_err)
    _check(lib().packed_scatter(B, D, pt, n_pt, reqs.data_ptr(), _n_reqs(reqs), err, _stream(stream)))


def kvx_gather_slice(src, src_spec, dst, buf_spec, sl, src_pt, reqs, dev_err=None,
                     stream=None) -> None:
    """Slice of a pool -> flat buffer holding exactly the slice (see
    kvx_gather_slice in include/kvx.h).  ``sl`` is a ``Slice`` or the nine
    range fields."""
    S, B = _pool_arg(src_spec, src, "src"), _buf_arg(buf_spec, dst, "dst")
    X = _slice_arg(sl)
    pt, n_pt = _table(src_pt, "src_pt")
    err = _err_word(dev_err)
    _check(lib().packed_gather_slice(S, B, X, pt, n_pt, reqs.data_ptr(), _n_reqs(reqs), err, _stream(stream)))


def kvx_scatter_slice(src, buf_spec, dst, dst_spec, sl, dst_pt, reqs, dev_err=None,
                      stream=None) -> None:
    """Flat buffer holding exactly a slice -> that slice of a pool (see
    kvx_scatter_slice in include/kvx.h)."""
    B, D = _buf_arg(buf_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    X = _slice_arg(sl)
    pt, n_pt = _table(dst_pt, "dst_pt")
    err = _err_word(dev_err)
    _check(lib().packed_scatter_slice(B, D, X, pt, n_pt, reqs.data_ptr(), _n_reqs(reqs), err,
                                      _stream(stream)))


def pack_hash_reqs(rows) -> np.ndarray:
    """(payload_off, out_off, seed, n_positions) rows -> kvx_hash_req records."""
    rows = list(rows)
    out = np.zeros(len(rows), dtype=HASH_REQ_DTYPE)
    for i, (po, oo, seed, n) in enumerate(rows):
        out[i] = (int(po), int(oo), int(seed) & 0xFFFFFFFFFFFFFFFF, int(n), 0)
    return out


def device_hash_reqs(rows, device="cuda"):
    import torch
    return torch.from_numpy(pack_hash_reqs(rows).view(np.uint8).copy()).to(device)


def kvx_page_hashes(payload, rec_bytes, page_tokens, reqs, out, dev_err, stream=None,
                    library=None) -> None:
    """Chained page hashes (see kvx_page_hashes in include/kvx.h).  ``payload``
    is a device tensor of records of ``rec_bytes`` bytes, ``reqs`` a device
    tensor from ``device_hash_reqs``, ``out`` a 64-bit device tensor (one
    word per page) and ``dev_err`` the device error word the call requires.
    ``library`` is a build loaded with ``load`` (default: ``lib()``)."""
    nbytes = payload.numel() * payload.element_size()
    if nbytes % rec_bytes:
        raise ValueError("payload is not a whole number of records")
    if out.element_size() != 8 or not out.is_contiguous() or not payload.is_contiguous():
        raise ValueError("out must be a contiguous 64-bit tensor; payload contiguous")
    _err_word(dev_err)
    rb = reqs.numel() * reqs.element_size()
    if rb % HASH_REQ_DTYPE.itemsize:
        raise ValueError("reqs must hold whole 32-byte kvx_hash_req records")
    if not reqs.is_contiguous():
        raise ValueError("reqs must be contiguous")
    L = library or lib()
    status = L.kvx_page_hashes(_ptr(payload), nbytes // rec_bytes, int(rec_bytes),
                               int(page_tokens), _ptr(reqs), rb // HASH_REQ_DTYPE.itemsize,
                               _ptr(out), out.numel(), _ptr(dev_err), _stream(stream))
    if status != 0:
        raise KvxError(status, L.kvx_last_error().decode())


def kvx_strerror(status: int) -> str:
    return lib().kvx_strerror(status).decode()


def kvx_last_error() -> str:
    return lib().kvx_last_error().decode()


def kvx_abi_version() -> int:
    return int(lib().kvx_abi_version())


# Launch choice of planned transfers and launch kinds (include/kvx.h).
CHOOSE_MEASURED, CHOOSE_SWEEP, CHOOSE_GRID = 0, 1, 2
LAUNCH_NONE, LAUNCH_GRID, LAUNCH_SWEEP = 0, 1, 2
LAUNCH_NAMES = {LAUNCH_NONE: "none", LAUNCH_GRID: "grid", LAUNCH_SWEEP: "sweep"}


def kvx_set_launch_choice(mode: int, library=None) -> None:
    """How planned transfers that can sweep pick their launch: CHOOSE_MEASURED,
    CHOOSE_SWEEP or CHOOSE_GRID (process-wide; forgets earlier measurements)."""
    L = library or lib()
    status = L.kvx_set_launch_choice(int(mode))
    if status != 0:
        raise KvxError(status, L.kvx_last_error().decode())


def kvx_launch_choice(library=None) -> int:
    return int((library or lib()).kvx_launch_choice())


def kvx_last_launch(library=None) -> int:
    """LAUNCH_NONE, LAUNCH_GRID or LAUNCH_SWEEP: the kind of the last kernel
    this thread's last copy call enqueued."""
    return int((library or lib()).kvx_last_launch())


# ---------------------------------------------------------------------------
# a decode step over a paged cache
# ---------------------------------------------------------------------------

APPEND_REQ_DTYPE = np.dtype([("pt_off", "<i8"), ("row_off", "<i8"), ("start", "<i4"), ("position", "<i4"),
                             ("n_tokens", "<i4"), ("reserved", "<i4")])
ATTEND_REQ_DTYPE = np.dtype([("pt_off", "<i8"), ("acc_off", "<i8"), ("start", "<i4"), ("end", "<i4")])
SELECT_REQ_DTYPE = np.dtype([("acc_off", "<i8"), ("kept_off", "<i8"), ("out_off", "<i8"), ("n_tokens", "<i4"),
                             ("n_keep", "<i4"), ("sink", "<i4"), ("recent", "<i4")])


def _pack(rows, dtype) -> np.ndarray:
    """Rows with a column per field of ``dtype`` (but ``reserved``) as records."""
    names = [n for n in dtype.names if n != "reserved"]
    rows = np.asarray(rows, dtype=np.int64).reshape(-1, len(names))
    out = np.zeros(len(rows), dtype=dtype)
    for i, name in enumerate(names):
        col = rows[:, i]
        if dtype[name].itemsize == 4 and ((col < -2**31) | (col >= 2**31)).any():
            raise ValueError(f"{name} does not fit int32")
        out[name] = col
    return out


def _device(records, device):
    import torch
    return torch.from_numpy(records.view(np.uint8).copy()).to(device)


def device_append_reqs(rows, device="cuda"):
    """(pt_off, row_off, start, position, n_tokens) rows as kvx_append_req
    records on the device."""
    return _device(_pack(rows, APPEND_REQ_DTYPE), device)


def device_attend_reqs(rows, device="cuda"):
    """(pt_off, acc_off, start, end) rows as kvx_attend_req records on the device."""
    return _device(_pack(rows, ATTEND_REQ_DTYPE), device)


def device_select_reqs(rows, device="cuda"):
    """(acc_off, kept_off, out_off, n_tokens, n_keep, sink, recent) rows as
    kvx_select_req records on the device."""
    return _device(_pack(rows, SELECT_REQ_DTYPE), device)


@dataclass(frozen=True)
class Rope:
    """A rotation (kvx_rope): ``freq`` a float32 device tensor of radians per
    position, one for each rotated pair of a head; ``rot_off`` the first
    rotated dimension; ``interleaved`` pairs (2j, 2j + 1) instead of (j, j +
    pairs); ``amplitude`` a factor on the rotated values."""
    freq: Any
    rot_off: int = 0
    interleaved: bool = False
    amplitude: float = 1.0


def rope_frequencies(rot_dim: int, base: float = 10000.0, factor: float = 1.0, scaling: str = "linear",
                     trained: int = 0, fast: float = 32.0, slow: float = 1.0):
    """(frequencies, amplitude) for ``Rope``: base ** (-2j / rot_dim) for the
    rot_dim / 2 pairs, as a float32 numpy array, stretched for contexts
    ``factor`` times as long as the trained ones:
    - "linear": every frequency divided by factor;
    - "base": the base raised to base * factor ** (rot_dim / (rot_dim - 2)), which
      leaves the first frequency and divides the last by factor;
    - "ramp": pairs that turn more than ``fast`` times within the ``trained``
      length stay, those that turn less than ``slow`` times are divided by
      factor, linearly in the pair's index between (from the last index, or 0,
      to the first whose pair turns at least `fast` and at most `slow` times);
      the amplitude is 0.1 ln(factor) + 1."""
    if rot_dim < 2 or rot_dim % 2 or base <= 1 or factor < 1:
        raise ValueError("rot_dim must be even and >= 2, base above 1 and factor >= 1")
    j = np.arange(0, rot_dim, 2, dtype=np.float64)
    freq = base ** (-j / rot_dim)
    if scaling == "linear":
        return (freq / factor).astype(np.float32), 1.0
    if scaling == "base":
        if rot_dim < 4:
            raise ValueError("scaling 'base' needs rot_dim >= 4")
        return ((base * factor ** (rot_dim / (rot_dim - 2))) ** (-j / rot_dim)).astype(np.float32), 1.0
    if scaling != "ramp":
        raise ValueError(f"scaling must be 'linear', 'base' or 'ramp' (got {scaling!r})")
    if trained < 1 or fast <= slow or slow <= 0:
        raise ValueError("scaling 'ramp' needs the trained length and fast > slow > 0")

    def pair(turns):                   # the (real) pair index that turns so often within `trained`
        return rot_dim * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(base))
    # The ends are those of the turns, wherever the last pair is: it may turn more often than `slow`.
    lo, hi = max(0, math.floor(pair(fast))), math.ceil(pair(slow))
    keep = np.clip((hi - j / 2) / (hi - lo), 0, 1) if hi > lo else np.zeros_like(j)     # hi <= 0: none turns `slow` times
    return (freq * keep + freq / factor * (1 - keep)).astype(np.float32), 0.1 * math.log(factor) + 1


_ROWS_PACK = struct.Struct("=Q3q4i").pack
_ROPE_PACK = struct.Struct("=Q3if").pack
_ROW_TYPES: dict = {}


def _rows_arg(t, name: str) -> bytes:
    """The kvx_rows of a [rows, heads, head_dim] tensor of 16-bit values,
    packed; its last dimension must be contiguous."""
    if not _ROW_TYPES:
        import torch
        _ROW_TYPES.update({torch.bfloat16: 0, torch.float16: 1})
    code = _ROW_TYPES.get(t.dtype)
    if code is None or t.dim() != 3:
        raise ValueError(f"{name} must be a bfloat16 or float16 tensor [rows, heads, head_dim] "
                         f"(got {t.dtype}, {t.dim()} dimensions)")
    n, heads, d = t.shape
    s_row, s_head, s_d = t.stride()
    if s_d != 1 and d != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    # the stride of a dimension of one is never used, and torch leaves any value there
    return _ROWS_PACK(t.data_ptr(), n, s_row if n > 1 else 0, s_head if heads > 1 else 0, heads, d, code, 0)


def _floats(t, name: str):
    """The address and length of an optional contiguous float32 tensor."""
    if t is None:
        return None, 0
    if t.element_size() != 4 or not t.is_floating_point() or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor (got {t.dtype})")
    return t.data_ptr(), t.numel()


def _scales(t, spec):
    if t is None:
        return None
    ptr, n = _floats(t, "scales")
    if n != spec.C * spec.H:
        raise ValueError(f"scales holds {n} values, the pool has {spec.C} x {spec.H}")
    return ptr


def _reqs_arg(reqs, dtype):
    """The address and count of a tensor of records."""
    n, rest = divmod(reqs.nbytes, dtype.itemsize)
    if rest or not reqs.is_contiguous():
        raise ValueError(f"reqs must be contiguous and hold whole records of {dtype.itemsize} bytes")
    return reqs.data_ptr(), n


def kvx_append(pool, spec, layer, k, v, pt, reqs, max_tokens, q=None, q_out=None, rope=None, scales=None,
               dev_err=None, stream=None) -> None:
    """New tokens' keys and values into their pages, rotated, and their
    queries rotated (see kvx_append in include/kvx.h).  ``k``, ``v``, ``q`` and
    ``q_out`` are [rows, heads, head_dim] tensors (slices of a fused projection
    will do), ``v`` None for a pool of C 1; ``rope`` a ``Rope`` or None;
    ``scales`` a float32 tensor [C, H] for an e4m3 pool (e 1)."""
    P = _pool_arg(spec, pool, "pool")
    table, n_pt = _table(pt, "pt")
    rec, n = _reqs_arg(reqs, APPEND_REQ_DTYPE)
    R = None
    if rope is not None:
        f, pairs = _floats(rope.freq, "rope.freq")
        R = _ROPE_PACK(f or 0, 2 * pairs, int(rope.rot_off), int(bool(rope.interleaved)), float(rope.amplitude))
    _check(lib().kvx_append(P, int(layer), _scales(scales, spec), None if q is None else _rows_arg(q, "q"),
                            None if q_out is None else _rows_arg(q_out, "q_out"), _rows_arg(k, "k"),
                            None if v is None else _rows_arg(v, "v"), R, table, n_pt, rec, n, int(max_tokens),
                            _err_word(dev_err), _stream(stream)))


def attend_workspace_bytes(spec, n_reqs: int, q_heads: int, max_tokens: int, v_dim=None,
                           accumulate: bool = False) -> int:
    """kvx_attend_workspace for a pool shape; ``v_dim`` defaults to head_dim."""
    n = int(lib().kvx_attend_workspace(bytes(pool_desc(spec, 0)), int(n_reqs), int(q_heads),
                                       int(spec.D if v_dim is None else v_dim), int(max_tokens), int(bool(accumulate))))
    if n < 0:
        raise KvxError(-5, lib().kvx_last_error().decode())
    return n


def attend_workspace(spec, n_reqs: int, q_heads: int, max_tokens: int, v_dim=None, accumulate: bool = False,
                     device="cuda"):
    """A workspace for kvx_attend calls of up to ``n_reqs`` records and
    ``max_tokens`` positions: device memory, whatever it holds."""
    import torch
    return torch.empty(attend_workspace_bytes(spec, n_reqs, q_heads, max_tokens, v_dim, accumulate),
                       dtype=torch.uint8, device=device)


def _stride(stride, name: str, of, rows: int) -> int:
    """The stride of an optional array's rows, which only a single row or no array does without."""
    if stride is None:
        if of is not None and rows > 1:
            raise ValueError(f"{name} is needed for {rows} rows")
        return 0
    return int(stride)


def kvx_attend(q, out, pool, spec, layer, pt, reqs, max_tokens, workspace, scale=None, scales=None, lse=None,
               acc=None, acc_stride=None, dev_err=None, stream=None) -> None:
    """Attention of one query per record over a layer's pages (see kvx_attend
    in include/kvx.h).  ``q`` [records, q heads, head_dim] and ``out``
    [records, q heads, v_dim]; ``scale`` defaults to head_dim ** -0.5;
    ``workspace`` from ``attend_workspace``; ``lse`` and ``acc`` optional float32
    tensors, ``acc_stride`` the accumulators from one cache head to the next."""
    acc_stride = _stride(acc_stride, "acc_stride", acc, spec.H)
    P = _pool_arg(spec, pool, "pool")
    table, n_pt = _table(pt, "pt")
    rec, n = _reqs_arg(reqs, ATTEND_REQ_DTYPE)
    lse_ptr, n_lse = _floats(lse, "lse")
    if lse is not None and n_lse < n * q.shape[1]:
        raise ValueError(f"lse holds {n_lse} values, {n} records x {q.shape[1]} heads need more")
    acc_ptr, n_acc = _floats(acc, "acc")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _check(lib().kvx_attend(P, int(layer), _scales(scales, spec), _rows_arg(q, "q"), _rows_arg(out, "out"), lse_ptr,
                            float(spec.D ** -0.5 if scale is None else scale), table, n_pt, rec, n, int(max_tokens),
                            acc_ptr, n_acc, acc_stride, workspace.data_ptr(), workspace.nbytes,
                            _err_word(dev_err), _stream(stream)))


def kvx_select_kept(acc, acc_stride, rows, reqs, max_tokens, kept, kept_stride, acc_out=None, acc_out_stride=None,
                    dev_err=None, stream=None) -> None:
    """The positions that each of ``rows`` lists of every record keeps, by
    accumulated weight (see kvx_select_kept in include/kvx.h): ``acc`` and
    ``acc_out`` float32, ``kept`` an int32 tensor."""
    acc_out_stride = _stride(acc_out_stride, "acc_out_stride", acc_out, rows)
    a, n_a = _floats(acc, "acc")
    o, n_o = _floats(acc_out, "acc_out")
    kp, n_k = _table(kept, "kept")
    rec, n = _reqs_arg(reqs, SELECT_REQ_DTYPE)
    _check(lib().kvx_select_kept(a, n_a, int(acc_stride), int(rows), rec, n, int(max_tokens), kp, n_k,
                                 int(kept_stride), o, n_o, acc_out_stride, _err_word(dev_err), _stream(stream)))


def kvx_transfer_kept(src, src_spec, dst, dst_spec, src_pt, dst_pt, reqs, max_tokens, kept, kept_stride, sl=None,
                      dev_err=None, stream=None) -> None:
    """Listed positions of every layer and head, pool -> pool (see
    kvx_transfer_kept in include/kvx.h); ``reqs`` from ``device_reqs``, whose
    buf_off is the record's first list in ``kept``; ``sl`` an optional slice."""
    S, D = _pool_arg(src_spec, src, "src"), _pool_arg(dst_spec, dst, "dst")
    X = None if sl is None else _slice_arg(sl)
    spt, n_spt = _table(src_pt, "src_pt")
    dpt, n_dpt = _table(dst_pt, "dst_pt")
    kp, n_k = _table(kept, "kept")
    _check(lib().kvx_transfer_kept(S, D, X, spt, n_spt, dpt, n_dpt, reqs.data_ptr(), _n_reqs(reqs), int(max_tokens),
                                   kp, n_k, int(kept_stride), _err_word(dev_err), _stream(stream)))


# ---------------------------------------------------------------------------
# several tokens of a request
# ---------------------------------------------------------------------------

QUERIES_REQ_DTYPE = np.dtype([("pt_off", "<i8"), ("row_off", "<i8"), ("start", "<i4"), ("end", "<i4"),
                              ("n_queries", "<i4"), ("prefix", "<i4")])
PATH_REQ_DTYPE = np.dtype([("pt_off", "<i8"), ("path_off", "<i8"), ("start", "<i4"), ("n_tokens", "<i4")])
MAX_DRAFTS = 64

_NORM_PACK = struct.Struct("=Q2ifi").pack
_POSITIONS_PACK = struct.Struct("=QqQ2i").pack
_SCORES_PACK = struct.Struct("=Q2f2i").pack


def device_queries_reqs(rows, device="cuda"):
    """(pt_off, row_off, start, end, n_queries, prefix) rows as kvx_queries_req
    records on the device."""
    return _device(_pack(rows, QUERIES_REQ_DTYPE), device)


def device_path_reqs(rows, device="cuda"):
    """(pt_off, path_off, start, n_tokens) rows as kvx_path_req records on the device."""
    return _device(_pack(rows, PATH_REQ_DTYPE), device)


@dataclass(frozen=True)
class Norm:
    """A norm of each head (kvx_norm): ``weight`` a float32 device tensor of
    factors, one for each normed element from ``off`` on; None for factors of
    1, with ``dim`` elements.  A model that stores its factors less one adds
    the one when it loads them."""
    weight: Any = None
    off: int = 0
    eps: float = 1e-6
    dim: int = 0


def _norm_arg(norm, name: str):
    if norm is None:
        return None
    ptr, n = _floats(norm.weight, name + ".weight")
    if norm.weight is not None and norm.dim not in (0, n):
        raise ValueError(f"{name}: dim {norm.dim}, but {n} weights")
    return _NORM_PACK(ptr or 0, n if norm.weight is not None else int(norm.dim), int(norm.off), float(norm.eps), 0)


def _positions_arg(positions, axis, k, rope):
    """The kvx_positions of an int32 tensor [rows] or [axes, rows] and an optional
    int32 tensor of each pair's axis."""
    if positions is None:
        if axis is not None:
            raise ValueError("axis is given without positions")
        return None
    if positions.element_size() != 4 or positions.is_floating_point() or positions.dim() not in (1, 2):
        raise ValueError(f"positions must be an int32 tensor [rows] or [axes, rows] (got {positions.dtype})")
    axes = positions.shape[0] if positions.dim() == 2 else 1
    if positions.shape[-1] != k.shape[0] or (positions.shape[-1] > 1 and positions.stride(-1) != 1):
        raise ValueError(f"positions must have contiguous entries for k's {k.shape[0]} rows")
    a, n = None, 0
    if axis is not None:
        a, n = _table(axis, "axis")
        if rope is None or n != rope.freq.numel():
            raise ValueError(f"axis holds {n} entries: one for each rotated pair is needed")
    stride = positions.stride(0) if positions.dim() == 2 and axes > 1 else 0
    return _POSITIONS_PACK(positions.data_ptr(), stride, a or 0, axes, 0)


def kvx_append_normed(pool, spec, layer, k, v, pt, reqs, max_tokens, q=None, q_out=None, rope=None, q_norm=None,
                      k_norm=None, positions=None, axis=None, scales=None, dev_err=None, stream=None) -> None:
    """kvx_append with queries and keys normed per head before they are rotated,
    and with positions of their own (see kvx_append_normed in include/kvx.h).
    ``q_norm`` and ``k_norm`` a ``Norm`` or None; ``positions`` an int32 device
    tensor [rows] or [axes, rows] or None (those of the records); ``axis`` an
    int32 device tensor with the axis of each rotated pair, None for all on axis
    0; everything else as ``kvx_append``."""
    P = _pool_arg(spec, pool, "pool")
    table, n_pt = _table(pt, "pt")
    rec, n = _reqs_arg(reqs, APPEND_REQ_DTYPE)
    R = None
    if rope is not None:
        f, pairs = _floats(rope.freq, "rope.freq")
        R = _ROPE_PACK(f or 0, 2 * pairs, int(rope.rot_off), int(bool(rope.interleaved)), float(rope.amplitude))
    _check(lib().kvx_append_normed(P, int(layer), _scales(scales, spec), None if q is None else _rows_arg(q, "q"),
                                   None if q_out is None else _rows_arg(q_out, "q_out"), _rows_arg(k, "k"),
                                   None if v is None else _rows_arg(v, "v"), R, _norm_arg(q_norm, "q_norm"),
                                   _norm_arg(k_norm, "k_norm"), _positions_arg(positions, axis, k, rope), table, n_pt, rec, n,
                                   int(max_tokens), _err_word(dev_err), _stream(stream)))


@dataclass(frozen=True)
class Scores:
    """What becomes of q . k (kvx_scores): ``scale`` (None: head_dim ** -0.5),
    ``cap`` (cap * tanh(s / cap); 0: none), ``slopes`` a float32 device tensor, one
    for each query head, of a bias -slope * distance, ``window`` the positions seen
    from a query back, its own included (0: all)."""
    scale: Any = None
    cap: float = 0.0
    slopes: Any = None
    window: int = 0


def queries_workspace_bytes(spec, n_reqs: int, q_heads: int, max_queries: int, max_tokens: int, v_dim=None) -> int:
    """kvx_queries_workspace for a pool shape; ``v_dim`` defaults to head_dim."""
    n = int(lib().kvx_queries_workspace(bytes(pool_desc(spec, 0)), int(n_reqs), int(q_heads),
                                        int(spec.D if v_dim is None else v_dim), int(max_queries), int(max_tokens)))
    if n < 0:
        raise KvxError(-5, lib().kvx_last_error().decode())
    return n


def queries_workspace(spec, n_reqs: int, q_heads: int, max_queries: int, max_tokens: int, v_dim=None, device="cuda"):
    """A workspace for kvx_attend_prompt and kvx_attend_tree calls of up to
    ``n_reqs`` records, ``max_queries`` queries and ``max_tokens`` positions each:
    device memory, whatever it holds."""
    import torch
    return torch.empty(queries_workspace_bytes(spec, n_reqs, q_heads, max_queries, max_tokens, v_dim), dtype=torch.uint8,
                       device=device)


def _attend_queries(q, out, pool, spec, layer, pt, reqs, tree, max_queries, max_tokens, workspace, scores, scales, lse,
                    dev_err, stream):
    P = _pool_arg(spec, pool, "pool")
    table, n_pt = _table(pt, "pt")
    rec, n = _reqs_arg(reqs, QUERIES_REQ_DTYPE)
    lse_ptr, n_lse = _floats(lse, "lse")
    if lse is not None and n_lse < q.shape[0] * q.shape[1]:
        raise ValueError(f"lse holds {n_lse} values, {q.shape[0]} rows x {q.shape[1]} heads need more")
    s = scores or Scores()
    slopes, n_slopes = _floats(s.slopes, "slopes")
    if s.slopes is not None and n_slopes != q.shape[1]:
        raise ValueError(f"slopes holds {n_slopes} values for {q.shape[1]} query heads")
    if tree is not None and (tree.element_size() != 8 or tree.is_floating_point() or not tree.is_contiguous()
                             or tree.numel() < q.shape[0]):
        raise ValueError(f"tree must be a contiguous 64-bit integer tensor with an entry for each of {q.shape[0]} rows")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    X = _SCORES_PACK(slopes or 0, float(spec.D ** -0.5 if s.scale is None else s.scale), float(s.cap), int(s.window), 0)
    head = (P, int(layer), _scales(scales, spec), _rows_arg(q, "q"), _rows_arg(out, "out"), lse_ptr, X, table, n_pt, rec)
    rest = (n, int(max_queries), int(max_tokens), workspace.data_ptr(), workspace.nbytes, _err_word(dev_err),
            _stream(stream))
    if tree is None:
        return _check(lib().kvx_attend_prompt(*head, *rest))
    _check(lib().kvx_attend_tree(*head, tree.data_ptr(), *rest))


def kvx_attend_prompt(q, out, pool, spec, layer, pt, reqs, max_queries, max_tokens, workspace, scores=None, scales=None,
                      lse=None, dev_err=None, stream=None) -> None:
    """Attention of the last queries of each record's positions over a layer's
    pages (see kvx_attend_prompt in include/kvx.h).  ``q`` [rows, q heads,
    head_dim] and ``out`` [rows, q heads, v_dim]; ``reqs`` from
    ``device_queries_reqs``; ``scores`` a ``Scores``; ``workspace`` from
    ``queries_workspace``; ``lse`` an optional float32 tensor [rows, q heads]."""
    _attend_queries(q, out, pool, spec, layer, pt, reqs, None, max_queries, max_tokens, workspace, scores, scales, lse,
                    dev_err, stream)


def kvx_attend_tree(q, out, pool, spec, layer, pt, reqs, tree, max_queries, max_tokens, workspace, scores=None,
                    scales=None, lse=None, dev_err=None, stream=None) -> None:
    """Attention of drafted tokens that form a tree (see kvx_attend_tree in
    include/kvx.h): ``tree`` a 64-bit integer device tensor, for each row the bits
    of the drafts that it sees, its ancestors and itself; everything else as
    ``kvx_attend_prompt``."""
    if tree is None:
        raise ValueError("tree is needed")
    _attend_queries(q, out, pool, spec, layer, pt, reqs, tree, max_queries, max_tokens, workspace, scores, scales, lse,
                    dev_err, stream)


def kvx_keep_path(pool, spec, pt, reqs, max_tokens, path, dev_err=None, stream=None) -> None:
    """Accepted drafts' rows to the front of the drafts' slots, in every layer, in
    place (see kvx_keep_path in include/kvx.h): ``reqs`` from
    ``device_path_reqs``, ``path`` an int32 tensor of their ascending lists."""
    P = _pool_arg(spec, pool, "pool")
    table, n_pt = _table(pt, "pt")
    rec, n = _reqs_arg(reqs, PATH_REQ_DTYPE)
    pp, n_path = _table(path, "path")
    _check(lib().kvx_keep_path(P, table, n_pt, rec, n, int(max_tokens), pp, n_path, _err_word(dev_err), _stream(stream)))
