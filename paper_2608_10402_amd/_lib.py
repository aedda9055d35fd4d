"""ctypes binding of libtide.so: the entry points of include/tide.h under the same names.

Argument marshalling only -- every step of the computation runs in the HIP kernels.
Device buffers are torch tensors on a ROCm device (torch supplies memory and streams);
lengths are host arrays.  Missing library => ImportError; a non-zero status from the
library => TideError.  There is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtide.so")

TIDE_OK = 0
TIDE_ERR_INVALID_ARG = -1
TIDE_ERR_UNSUPPORTED = -2
TIDE_ERR_CAPACITY = -3
TIDE_ERR_HIP = -4
TIDE_ERR_PAGE_RANGE = -5

TIDE_OP_KV_APPEND = 1
TIDE_OP_EXTEND = 2
TIDE_OP_DECODE = 3
TIDE_OP_FULL_PREFILL = 4
TIDE_OP_KV4_APPEND = 5
TIDE_OP_KV4_UNPACK = 6
TIDE_OP_KV4_DECODE = 7
TIDE_OP_KV4_EXTEND = 8
TIDE_OP_ATTN_MASS = 9
TIDE_OP_KV_EVICT = 10
TIDE_OP_SLOT_APPEND = 11
TIDE_OP_KEY_BOUNDS = 12
TIDE_OP_BLOCK_SELECT = 13
TIDE_OP_SPARSE_ATTN = 14

# bytes of the static device scratch of tide_decode_attn_noalloc (TIDE_NOALLOC_SCRATCH_BYTES)
NOALLOC_SCRATCH_BYTES = 64 << 20

EXPORTED = ("tide_workspace_size", "tide_kv_append", "tide_extend_attn", "tide_decode_attn",
            "tide_full_prefill_attn", "tide_decode_attn_shared", "tide_workspace_size_shared",
            "tide_decode_append_attn", "tide_decode_attn_noalloc", "tide_extend_append_attn",
            "tide_kv4_append", "tide_kv4_unpack", "tide_kv4_decode_attn",
            "tide_kv4_decode_append_attn", "tide_kv4_extend_attn", "tide_attn_mass",
            "tide_kv4_attn_mass", "tide_kv_evict", "tide_kv4_evict",
            "tide_rows_workspace_size", "tide_rows_workspace_bound", "tide_page_map", "tide_slot_append", "tide_key_bounds",
            "tide_block_select", "tide_sparse_attn",
            "tide_plan_info_get", "tide_ctb_create", "tide_ctb_step", "tide_ctb_get_stats", "tide_ctb_destroy",
            "tide_status_string", "tide_shutdown")


class TideError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, status_string(status), status))


class tide_dims(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("sm_scale", ctypes.c_float)]


class tide_plan_info(ctypes.Structure):
    _fields_ = [("num_items", ctypes.c_int32), ("waves_per_group", ctypes.c_int32),
                ("split", ctypes.c_int32), ("max_splits", ctypes.c_int32),
                ("merge_in_kernel", ctypes.c_int32), ("run_steps", ctypes.c_int32),
                ("workspace_bytes", ctypes.c_size_t)]


def make_dims(num_q_heads: int, num_kv_heads: int, head_dim: int, sm_scale: float,
              page_size: int = 16) -> tide_dims:
    return tide_dims(num_q_heads, num_kv_heads, head_dim, page_size, sm_scale)


_lib = None


def load(path: str = LIB_PATH):
    """Load libtide.so (once).  Raises ImportError when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError("libtide.so not found at %s; build it with "
                          "`python -m paper_2608_10402_amd.build`" % path)
    lib = ctypes.CDLL(path)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    dims_p = ctypes.POINTER(tide_dims)
    lib.tide_workspace_size.argtypes = [ctypes.c_int, i32, vp, vp, dims_p, i32,
                                        ctypes.POINTER(sz)]
    lib.tide_kv_append.argtypes = [vp, vp, vp, vp, i64, vp, i32, i32, vp, vp, dims_p, vp, sz, vp]
    lib.tide_extend_attn.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, vp, dims_p, vp, vp, vp,
                                     sz, vp]
    lib.tide_decode_attn.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, dims_p, i32, vp, vp, vp,
                                     sz, vp]
    lib.tide_full_prefill_attn.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, dims_p, vp, vp, vp,
                                           sz, vp]
    lib.tide_decode_append_attn.argtypes = [vp, vp, vp, vp, vp, i64, vp, i32, i32, vp, dims_p,
                                            i32, vp, vp, vp, sz, vp]
    lib.tide_extend_append_attn.argtypes = [vp, vp, vp, vp, vp, i64, vp, i32, i32, vp, vp, dims_p,
                                            vp, vp, vp, sz, vp]
    lib.tide_decode_attn_noalloc.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, dims_p, i32, vp,
                                             vp, vp]
    lib.tide_decode_attn_shared.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, i32, vp, vp, dims_p,
                                            i32, vp, vp, vp, sz, vp]
    lib.tide_workspace_size_shared.argtypes = [i32, vp, i32, vp, vp, dims_p, i32,
                                               ctypes.POINTER(sz)]
    lib.tide_kv4_append.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, vp, dims_p, vp, sz, vp]
    lib.tide_kv4_unpack.argtypes = [vp, i64, vp, i32, i32, vp, vp, dims_p, vp, vp, vp, sz, vp]
    lib.tide_kv4_decode_attn.argtypes = [vp, vp, i64, vp, i32, i32, vp, dims_p, vp, vp, vp, sz, vp]
    lib.tide_kv4_decode_append_attn.argtypes = [vp, vp, vp, vp, i64, vp, i32, i32, vp, dims_p, vp, vp,
                                                vp, sz, vp]
    lib.tide_kv4_extend_attn.argtypes = [vp, vp, i64, vp, i32, i32, vp, vp, dims_p, vp, vp, vp, sz,
                                         vp]
    lib.tide_attn_mass.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, vp, vp, dims_p, vp, vp, sz, vp]
    lib.tide_kv4_attn_mass.argtypes = lib.tide_attn_mass.argtypes
    lib.tide_kv_evict.argtypes = [vp, vp, vp, i64, vp, i32, vp, i32, i32, vp, vp, vp, dims_p, vp, vp,
                                  sz, vp]
    lib.tide_kv4_evict.argtypes = [vp, vp, i64, vp, i32, vp, i32, i32, vp, vp, vp, dims_p, vp, vp,
                                   sz, vp]
    lib.tide_rows_workspace_size.argtypes = [ctypes.c_int, i32, i32, i32, dims_p, ctypes.POINTER(sz)]
    lib.tide_rows_workspace_bound.argtypes = lib.tide_rows_workspace_size.argtypes
    lib.tide_page_map.argtypes = [vp, vp, i32, vp, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, dims_p,
                                  vp]
    lib.tide_slot_append.argtypes = [vp, vp, vp, i32, vp, vp, i64, vp, vp, dims_p, vp, sz, vp]
    lib.tide_key_bounds.argtypes = [vp, i64, vp, i32, i32, vp, vp, i32, vp, vp, dims_p, vp, sz, vp]
    lib.tide_block_select.argtypes = [vp, vp, vp, i32, vp, vp, i64, vp, i32, i32, i32, i32, i32, i32, dims_p,
                                      vp, vp, sz, vp]
    lib.tide_sparse_attn.argtypes = [vp, vp, vp, i64, vp, i32, i32, vp, vp, i32, vp, i32, dims_p, vp, vp, vp,
                                     sz, vp]
    lib.tide_plan_info_get.argtypes = [ctypes.c_int, i32, vp, vp, dims_p, i32,
                                       ctypes.POINTER(tide_plan_info)]
    lib.tide_ctb_create.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp, vp, vp,
                                    ctypes.POINTER(vp)]
    lib.tide_ctb_step.argtypes = [vp, vp]
    lib.tide_ctb_get_stats.argtypes = [vp, vp]
    lib.tide_ctb_destroy.argtypes = [vp]
    for name in EXPORTED[:-2]:
        getattr(lib, name).restype = ctypes.c_int
    lib.tide_status_string.argtypes = [ctypes.c_int]
    lib.tide_status_string.restype = ctypes.c_char_p
    lib.tide_shutdown.argtypes = []
    lib.tide_shutdown.restype = None
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().tide_status_string(int(status)).decode()


# ---- marshalling helpers ------------------------------------------------------------------
# A small call takes the host longer than the GPU (four tasks' decode step: about 15 us of
# kernels; 23 us of host time with 12 us of it in these checks, 16 us with 7 us), so a check is
# one or two attribute reads when it passes, and what went wrong is worked out only when it
# does not.
_I32 = np.dtype(np.int32)


def _dev(t, dtype, name, nullable=False):
    if isinstance(t, torch.Tensor):
        if t.is_cuda and t.dtype is dtype and t.is_contiguous():
            return t.data_ptr() if t.numel() else None
    elif t is None:
        if nullable:
            return None
        raise ValueError("%s is required" % name)
    else:
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.device.type != "cuda":
        raise ValueError("%s must live on a ROCm device" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    raise ValueError("%s must be contiguous" % name)


def _host(a, name):
    if a is None:
        return None, None
    arr = a
    if type(a) is not np.ndarray or a.dtype != _I32 or not a.flags.c_contiguous:
        arr = np.ascontiguousarray(np.asarray(a), dtype=np.int32)
    if arr.ndim != 1:
        raise ValueError("%s must be 1-D" % name)
    return arr, arr.__array_interface__["data"][0]


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:  # current_stream() without building its Stream object
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _check(status, where):
    if status != TIDE_OK:
        raise TideError(status, where)


def _ws(workspace):
    if workspace is None:
        return None, 0
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda:
        raise ValueError("workspace must be a device tensor")
    return workspace.data_ptr(), workspace.nbytes


def _same_device(*tensors):
    """All device tensors of one call must live on one device (the pointers are handed to
    kernels launched on that device)."""
    first = None
    for t in tensors:
        if isinstance(t, torch.Tensor):
            d = t.get_device()
            if first is None:
                first = d
            elif d != first:
                devs = {t.device for t in tensors if isinstance(t, torch.Tensor)}
                raise ValueError("all tensors of a call must be on one device, got %s"
                                 % sorted(map(str, devs)))


def _rows(t, name, rows, heads, d):
    """t must be [rows][heads][d] (the library reads and writes exactly that many bytes).
    rows None: the lengths are invalid, which the library itself rejects before any device
    work."""
    if t is None or rows is None:
        return
    if t.shape != (rows, heads, d):
        raise ValueError("%s must have shape (%d, %d, %d), got %s"
                         % (name, rows, heads, d, tuple(t.shape)))


def _lse(t, rows, heads):
    if t is not None and rows is not None and t.shape != (rows, heads):
        raise ValueError("lse must have shape (%d, %d), got %s" % (rows, heads, tuple(t.shape)))


def _block_table(bt, num_tasks):
    if not isinstance(bt, torch.Tensor) or bt.dim() != 2:
        raise ValueError("block_table must be a 2-D tensor [num_tasks][bt_stride]")
    rows, stride = bt.shape
    if rows < num_tasks or stride < 1:
        raise ValueError("block_table has %d rows for %d tasks" % (rows, num_tasks))
    return stride


def _lens_total(lens):
    """Sum of a host length array (the row count the library will use), or None when a
    length is negative: the library returns TIDE_ERR_INVALID_ARG for that itself."""
    if lens is None:
        return None
    if lens.size <= 512:
        values = lens.tolist()
        return sum(values) if not values or min(values) >= 0 else None
    return None if (lens < 0).any() else int(lens.sum(dtype=np.int64))


def rows_of(lens) -> int:
    """Packed rows of these per-task counts (0 for counts that the library will refuse)."""
    arr, _ = _host(lens, "lens")
    return (_lens_total(arr) or 0) if arr is not None else 0


def _pool_shape(k_pool, v_pool, dims):
    shape = k_pool.shape
    if len(shape) != 4 or v_pool.dim() != 4:
        raise ValueError("pools must be 4-D")
    if shape[1:] != (dims.num_kv_heads, dims.page_size, dims.head_dim):
        raise ValueError("k_pool must be [num_pages][Hkv][page_size][d]")
    if v_pool.shape != shape:
        raise ValueError("v_pool must be [num_pages][Hkv][page_size][d]")
    return shape[0]


# ---- entry points ---------------------------------------------------------------------------
def tide_workspace_size(op: int, lens_a, lens_b, dims: tide_dims, num_splits: int = 0) -> int:
    a, a_p = _host(lens_a, "lens_a")
    b, b_p = _host(lens_b, "lens_b")
    n = 0 if a is None else int(a.size)
    out = ctypes.c_size_t(0)
    _check(load().tide_workspace_size(op, n, a_p, b_p, ctypes.byref(dims), int(num_splits),
                                      ctypes.byref(out)), "tide_workspace_size")
    return int(out.value)


def tide_plan_info_get(op: int, lens_a, lens_b, dims: tide_dims, num_splits: int = 0) -> dict:
    """The launch a call with these lengths makes (items, waves per workgroup, ...)."""
    a, a_p = _host(lens_a, "lens_a")
    b, b_p = _host(lens_b, "lens_b")
    n = 0 if a is None else int(a.size)
    info = tide_plan_info()
    _check(load().tide_plan_info_get(op, n, a_p, b_p, ctypes.byref(dims), int(num_splits),
                                     ctypes.byref(info)), "tide_plan_info_get")
    return {name: getattr(info, name) for name, _ in tide_plan_info._fields_}


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(1, int(nbytes)), dtype=torch.uint8, device=device)


def tide_kv_append(k_new, v_new, k_pool, v_pool, block_table, prefix_lens, extend_lens,
                   dims: tide_dims, workspace, stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    p, p_p = _host(prefix_lens, "prefix_lens")
    e, e_p = _host(extend_lens, "extend_lens")
    if p is None or e is None or p.size != e.size:
        raise ValueError("prefix_lens and extend_lens must have one entry per task")
    rows = _lens_total(e)
    _rows(k_new, "k_new", rows, dims.num_kv_heads, dims.head_dim)
    _rows(v_new, "v_new", rows, dims.num_kv_heads, dims.head_dim)
    _block_table(block_table, int(p.size))
    _same_device(k_new, v_new, k_pool, v_pool, block_table, workspace)
    ws, ws_n = _ws(workspace)
    _check(load().tide_kv_append(
        _dev(k_new, torch.bfloat16, "k_new"), _dev(v_new, torch.bfloat16, "v_new"),
        _dev(k_pool, torch.bfloat16, "k_pool"), _dev(v_pool, torch.bfloat16, "v_pool"),
        num_pages, _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]),
        int(p.size), p_p, e_p, ctypes.byref(dims), ws, ws_n, _stream(stream)), "tide_kv_append")


def tide_extend_attn(q, k_pool, v_pool, block_table, prefix_lens, extend_lens, dims: tide_dims,
                     out, lse=None, workspace=None, stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    p, p_p = _host(prefix_lens, "prefix_lens")
    e, e_p = _host(extend_lens, "extend_lens")
    if p is None or e is None or p.size != e.size:
        raise ValueError("prefix_lens and extend_lens must have one entry per task")
    rows = _lens_total(e)
    _rows(q, "q", rows, dims.num_q_heads, dims.head_dim)
    _rows(out, "out", rows, dims.num_q_heads, dims.head_dim)
    _lse(lse, rows, dims.num_q_heads)
    _block_table(block_table, int(p.size))
    _same_device(q, k_pool, v_pool, block_table, out, lse, workspace)
    ws, ws_n = _ws(workspace)
    _check(load().tide_extend_attn(
        _dev(q, torch.bfloat16, "q"), _dev(k_pool, torch.bfloat16, "k_pool"),
        _dev(v_pool, torch.bfloat16, "v_pool"), num_pages,
        _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(p.size),
        p_p, e_p, ctypes.byref(dims), _dev(out, torch.bfloat16, "out"),
        _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n, _stream(stream)),
        "tide_extend_attn")


def _decode_checks(q, out, lse, block_table, kv, dims, *others):
    if kv is None:
        raise ValueError("kv_lens is required")
    n = int(kv.size)
    _rows(q, "q", n, dims.num_q_heads, dims.head_dim)
    _rows(out, "out", n, dims.num_q_heads, dims.head_dim)
    _lse(lse, n, dims.num_q_heads)
    _block_table(block_table, n)
    _same_device(q, out, lse, block_table, *others)


def tide_extend_append_attn(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens,
                            extend_lens, dims: tide_dims, out, lse=None, workspace=None,
                            stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    p, p_p = _host(prefix_lens, "prefix_lens")
    e, e_p = _host(extend_lens, "extend_lens")
    if p is None or e is None or p.size != e.size:
        raise ValueError("prefix_lens and extend_lens must have one entry per task")
    rows = _lens_total(e)
    _rows(q, "q", rows, dims.num_q_heads, dims.head_dim)
    _rows(out, "out", rows, dims.num_q_heads, dims.head_dim)
    _rows(k_new, "k_new", rows, dims.num_kv_heads, dims.head_dim)
    _rows(v_new, "v_new", rows, dims.num_kv_heads, dims.head_dim)
    _lse(lse, rows, dims.num_q_heads)
    _block_table(block_table, int(p.size))
    _same_device(q, k_new, v_new, k_pool, v_pool, block_table, out, lse, workspace)
    ws, ws_n = _ws(workspace)
    _check(load().tide_extend_append_attn(
        _dev(q, torch.bfloat16, "q"), _dev(k_new, torch.bfloat16, "k_new"),
        _dev(v_new, torch.bfloat16, "v_new"), _dev(k_pool, torch.bfloat16, "k_pool"),
        _dev(v_pool, torch.bfloat16, "v_pool"), num_pages,
        _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(p.size),
        p_p, e_p, ctypes.byref(dims), _dev(out, torch.bfloat16, "out"),
        _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n, _stream(stream)),
        "tide_extend_append_attn")


def tide_decode_attn(q, k_pool, v_pool, block_table, kv_lens, dims: tide_dims, out, lse=None,
                     num_splits: int = 0, workspace=None, stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    kv, kv_p = _host(kv_lens, "kv_lens")
    _decode_checks(q, out, lse, block_table, kv, dims, k_pool, v_pool, workspace)
    ws, ws_n = _ws(workspace)
    _check(load().tide_decode_attn(
        _dev(q, torch.bfloat16, "q"), _dev(k_pool, torch.bfloat16, "k_pool"),
        _dev(v_pool, torch.bfloat16, "v_pool"), num_pages,
        _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(kv.size),
        kv_p, ctypes.byref(dims), int(num_splits), _dev(out, torch.bfloat16, "out"),
        _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n, _stream(stream)),
        "tide_decode_attn")


def tide_decode_append_attn(q, k_new, v_new, k_pool, v_pool, block_table, kv_lens,
                            dims: tide_dims, out, lse=None, num_splits: int = 0,
                            workspace=None, stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    kv, kv_p = _host(kv_lens, "kv_lens")
    _decode_checks(q, out, lse, block_table, kv, dims, k_pool, v_pool, k_new, v_new, workspace)
    _rows(k_new, "k_new", int(kv.size), dims.num_kv_heads, dims.head_dim)
    _rows(v_new, "v_new", int(kv.size), dims.num_kv_heads, dims.head_dim)
    ws, ws_n = _ws(workspace)
    _check(load().tide_decode_append_attn(
        _dev(q, torch.bfloat16, "q"), _dev(k_new, torch.bfloat16, "k_new"),
        _dev(v_new, torch.bfloat16, "v_new"), _dev(k_pool, torch.bfloat16, "k_pool"),
        _dev(v_pool, torch.bfloat16, "v_pool"), num_pages,
        _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(kv.size),
        kv_p, ctypes.byref(dims), int(num_splits), _dev(out, torch.bfloat16, "out"),
        _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n, _stream(stream)),
        "tide_decode_append_attn")


def tide_decode_attn_noalloc(q, k_pool, v_pool, block_table, kv_lens, dims: tide_dims, out,
                             lse=None, num_splits: int = 0, stream=None) -> None:
    """tide_decode_attn without a workspace: runs in the library's static device scratch
    (NOALLOC_SCRATCH_BYTES per GPU); calls that overlap on one GPU race."""
    num_pages = _pool_shape(k_pool, v_pool, dims)
    kv, kv_p = _host(kv_lens, "kv_lens")
    _decode_checks(q, out, lse, block_table, kv, dims, k_pool, v_pool)
    _check(load().tide_decode_attn_noalloc(
        _dev(q, torch.bfloat16, "q"), _dev(k_pool, torch.bfloat16, "k_pool"),
        _dev(v_pool, torch.bfloat16, "v_pool"), num_pages,
        _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(kv.size),
        kv_p, ctypes.byref(dims), int(num_splits), _dev(out, torch.bfloat16, "out"),
        _dev(lse, torch.float32, "lse", nullable=True), _stream(stream)),
        "tide_decode_attn_noalloc")


def _groups(group_start, shared_lens):
    gs, gs_p = _host(group_start, "group_start")
    sh, sh_p = _host(shared_lens, "shared_lens")
    if gs is None or sh is None or gs.size != sh.size + 1:
        raise ValueError("group_start must have one entry more than shared_lens")
    return int(sh.size), gs, gs_p, sh, sh_p


def tide_workspace_size_shared(kv_lens, group_start, shared_lens, dims: tide_dims,
                               num_splits: int = 0) -> int:
    kv, kv_p = _host(kv_lens, "kv_lens")
    ng, gs, gs_p, sh, sh_p = _groups(group_start, shared_lens)
    out = ctypes.c_size_t(0)
    _check(load().tide_workspace_size_shared(int(kv.size), kv_p, ng, gs_p, sh_p,
                                             ctypes.byref(dims), int(num_splits),
                                             ctypes.byref(out)), "tide_workspace_size_shared")
    return int(out.value)


def tide_decode_attn_shared(q, k_pool, v_pool, block_table, kv_lens, group_start, shared_lens,
                            dims: tide_dims, out, lse=None, num_splits: int = 0, workspace=None,
                            stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    kv, kv_p = _host(kv_lens, "kv_lens")
    ng, gs, gs_p, sh, sh_p = _groups(group_start, shared_lens)
    _decode_checks(q, out, lse, block_table, kv, dims, k_pool, v_pool, workspace)
    ws, ws_n = _ws(workspace)
    _check(load().tide_decode_attn_shared(
        _dev(q, torch.bfloat16, "q"), _dev(k_pool, torch.bfloat16, "k_pool"),
        _dev(v_pool, torch.bfloat16, "v_pool"), num_pages,
        _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(kv.size),
        kv_p, ng, gs_p, sh_p, ctypes.byref(dims), int(num_splits),
        _dev(out, torch.bfloat16, "out"), _dev(lse, torch.float32, "lse", nullable=True), ws,
        ws_n, _stream(stream)), "tide_decode_attn_shared")


def tide_full_prefill_attn(q, k_pool, v_pool, block_table, seq_lens, dims: tide_dims, out,
                           lse=None, workspace=None, stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    s, s_p = _host(seq_lens, "seq_lens")
    if s is None:
        raise ValueError("seq_lens is required")
    rows = _lens_total(s)
    _rows(q, "q", rows, dims.num_q_heads, dims.head_dim)
    _rows(out, "out", rows, dims.num_q_heads, dims.head_dim)
    _lse(lse, rows, dims.num_q_heads)
    _block_table(block_table, int(s.size))
    _same_device(q, k_pool, v_pool, block_table, out, lse, workspace)
    ws, ws_n = _ws(workspace)
    _check(load().tide_full_prefill_attn(
        _dev(q, torch.bfloat16, "q"), _dev(k_pool, torch.bfloat16, "k_pool"),
        _dev(v_pool, torch.bfloat16, "v_pool"), num_pages,
        _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(s.size),
        s_p, ctypes.byref(dims), _dev(out, torch.bfloat16, "out"),
        _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n, _stream(stream)),
        "tide_full_prefill_attn")


# ---- the 4-bit cache, attention mass, eviction ------------------------------------------------
def kv4_block_bytes(head_dim: int) -> int:
    """Bytes of one (page, kv head) block of a 4-bit pool (TIDE_KV4_BLOCK_BYTES)."""
    return 17 * head_dim


def _pool4_shape(kv4_pool, dims):
    if kv4_pool.dim() != 3 or kv4_pool.shape[1:] != (dims.num_kv_heads,
                                                     kv4_block_bytes(dims.head_dim)):
        raise ValueError("kv4_pool must be [num_pages][Hkv][%d]" % kv4_block_bytes(dims.head_dim))
    return kv4_pool.shape[0]


def _per_task(lens, name, n):
    """A host length array with one entry per task, or nothing."""
    arr, ptr = _host(lens, name)
    if arr is not None and arr.size != n:
        raise ValueError("%s must have one entry per task" % name)
    return arr, ptr


def _pair(a, b, a_name, b_name):
    a, a_p = _host(a, a_name)
    b, b_p = _host(b, b_name)
    if a is None or b is None or a.size != b.size:
        raise ValueError("%s and %s must have one entry per task" % (a_name, b_name))
    return a, a_p, b, b_p


def _invoke(name, on, stream, *args):
    """Calls an entry point on the device of `on` (its stream, staging and launches), which need
    not be the current one."""
    fn = getattr(load(), name)
    dev = on.get_device()
    if dev < 0 or dev == torch.cuda.current_device():
        status = fn(*args, _raw_stream(dev) if stream is None and _raw_stream is not None and dev >= 0
                    else _stream(stream))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _stream(stream))
    if status != TIDE_OK:
        raise TideError(status, name)


def _mass_pool(mass, num_pages, dims):
    if mass.shape != (num_pages, dims.num_kv_heads, dims.page_size):
        raise ValueError("mass must be [num_pages][Hkv][page_size], got %s" % (tuple(mass.shape),))


def tide_kv4_append(k_new, v_new, kv4_pool, block_table, prefix_lens, extend_lens, dims: tide_dims,
                    workspace, stream=None) -> None:
    num_pages = _pool4_shape(kv4_pool, dims)
    p, p_p, e, e_p = _pair(prefix_lens, extend_lens, "prefix_lens", "extend_lens")
    rows = _lens_total(e)
    _rows(k_new, "k_new", rows, dims.num_kv_heads, dims.head_dim)
    _rows(v_new, "v_new", rows, dims.num_kv_heads, dims.head_dim)
    _block_table(block_table, int(p.size))
    _same_device(k_new, v_new, kv4_pool, block_table, workspace)
    ws, ws_n = _ws(workspace)
    _invoke("tide_kv4_append", kv4_pool, stream,
            _dev(k_new, torch.bfloat16, "k_new"), _dev(v_new, torch.bfloat16, "v_new"),
            _dev(kv4_pool, torch.uint8, "kv4_pool"), num_pages,
            _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(p.size),
            p_p, e_p, ctypes.byref(dims), ws, ws_n)


def tide_kv4_unpack(kv4_pool, block_table, prefix_lens, extend_lens, dims: tide_dims, k_out=None,
                    v_out=None, workspace=None, stream=None):
    """Returns (k_out, v_out), new ones where they are None."""
    num_pages = _pool4_shape(kv4_pool, dims)
    p, p_p, e, e_p = _pair(prefix_lens, extend_lens, "prefix_lens", "extend_lens")
    rows = _lens_total(e)
    if k_out is None:
        k_out = torch.empty((rows or 0, dims.num_kv_heads, dims.head_dim), dtype=torch.bfloat16,
                            device=kv4_pool.device)
    if v_out is None:
        v_out = torch.empty_like(k_out)
    _rows(k_out, "k_out", rows, dims.num_kv_heads, dims.head_dim)
    _rows(v_out, "v_out", rows, dims.num_kv_heads, dims.head_dim)
    _block_table(block_table, int(p.size))
    _same_device(k_out, v_out, kv4_pool, block_table, workspace)
    ws, ws_n = _ws(workspace)
    _invoke("tide_kv4_unpack", kv4_pool, stream,
            _dev(kv4_pool, torch.uint8, "kv4_pool"), num_pages,
            _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(p.size),
            p_p, e_p, ctypes.byref(dims), _dev(k_out, torch.bfloat16, "k_out"),
            _dev(v_out, torch.bfloat16, "v_out"), ws, ws_n)
    return k_out, v_out


def tide_kv4_decode_attn(q, kv4_pool, block_table, kv_lens, dims: tide_dims, out, lse=None,
                         workspace=None, stream=None) -> None:
    num_pages = _pool4_shape(kv4_pool, dims)
    kv, kv_p = _host(kv_lens, "kv_lens")
    _decode_checks(q, out, lse, block_table, kv, dims, kv4_pool, workspace)
    ws, ws_n = _ws(workspace)
    _invoke("tide_kv4_decode_attn", kv4_pool, stream,
            _dev(q, torch.bfloat16, "q"), _dev(kv4_pool, torch.uint8, "kv4_pool"), num_pages,
            _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(kv.size),
            kv_p, ctypes.byref(dims), _dev(out, torch.bfloat16, "out"),
            _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n)


def tide_kv4_decode_append_attn(q, k_new, v_new, kv4_pool, block_table, kv_lens, dims: tide_dims,
                                out, lse=None, workspace=None, stream=None) -> None:
    num_pages = _pool4_shape(kv4_pool, dims)
    kv, kv_p = _host(kv_lens, "kv_lens")
    _decode_checks(q, out, lse, block_table, kv, dims, kv4_pool, k_new, v_new, workspace)
    _rows(k_new, "k_new", int(kv.size), dims.num_kv_heads, dims.head_dim)
    _rows(v_new, "v_new", int(kv.size), dims.num_kv_heads, dims.head_dim)
    ws, ws_n = _ws(workspace)
    _invoke("tide_kv4_decode_append_attn", kv4_pool, stream,
            _dev(q, torch.bfloat16, "q"), _dev(k_new, torch.bfloat16, "k_new"),
            _dev(v_new, torch.bfloat16, "v_new"), _dev(kv4_pool, torch.uint8, "kv4_pool"),
            num_pages, _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]),
            int(kv.size), kv_p, ctypes.byref(dims), _dev(out, torch.bfloat16, "out"),
            _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n)


def tide_kv4_extend_attn(q, kv4_pool, block_table, prefix_lens, extend_lens, dims: tide_dims, out,
                         lse=None, workspace=None, stream=None) -> None:
    num_pages = _pool4_shape(kv4_pool, dims)
    p, p_p, e, e_p = _pair(prefix_lens, extend_lens, "prefix_lens", "extend_lens")
    rows = _lens_total(e)
    _rows(q, "q", rows, dims.num_q_heads, dims.head_dim)
    _rows(out, "out", rows, dims.num_q_heads, dims.head_dim)
    _lse(lse, rows, dims.num_q_heads)
    _block_table(block_table, int(p.size))
    _same_device(q, kv4_pool, block_table, out, lse, workspace)
    ws, ws_n = _ws(workspace)
    _invoke("tide_kv4_extend_attn", kv4_pool, stream,
            _dev(q, torch.bfloat16, "q"), _dev(kv4_pool, torch.uint8, "kv4_pool"), num_pages,
            _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(p.size),
            p_p, e_p, ctypes.byref(dims), _dev(out, torch.bfloat16, "out"),
            _dev(lse, torch.float32, "lse", nullable=True), ws, ws_n)


def _attn_mass(name, q, lse, pool, pool_type, num_pages, block_table, prefix_lens, extend_lens,
               dims, mass, counted_lens, workspace, stream):
    p, p_p, e, e_p = _pair(prefix_lens, extend_lens, "prefix_lens", "extend_lens")
    counted, c_p = _per_task(counted_lens, "counted_lens", int(p.size))  # (held for the call)
    rows = _lens_total(e)
    _rows(q, "q", rows, dims.num_q_heads, dims.head_dim)
    _lse(lse, rows, dims.num_q_heads)
    _mass_pool(mass, num_pages, dims)
    _block_table(block_table, int(p.size))
    _same_device(q, lse, pool, block_table, mass, workspace)
    ws, ws_n = _ws(workspace)
    _invoke(name, pool, stream,
            _dev(q, torch.bfloat16, "q"), _dev(lse, torch.float32, "lse"),
            _dev(pool, pool_type, "pool"), num_pages,
            _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), int(p.size),
            p_p, e_p, c_p, ctypes.byref(dims), _dev(mass, torch.float32, "mass"), ws, ws_n)


def tide_attn_mass(q, lse, k_pool, block_table, prefix_lens, extend_lens, dims: tide_dims, mass,
                   counted_lens=None, workspace=None, stream=None) -> None:
    _attn_mass("tide_attn_mass", q, lse, k_pool, torch.bfloat16, _pool_shape(k_pool, k_pool, dims),
               block_table, prefix_lens, extend_lens, dims, mass, counted_lens, workspace, stream)


def tide_kv4_attn_mass(q, lse, kv4_pool, block_table, prefix_lens, extend_lens, dims: tide_dims,
                       mass, counted_lens=None, workspace=None, stream=None) -> None:
    _attn_mass("tide_kv4_attn_mass", q, lse, kv4_pool, torch.uint8, _pool4_shape(kv4_pool, dims),
               block_table, prefix_lens, extend_lens, dims, mass, counted_lens, workspace, stream)


def _evict_lens(mass, num_pages, block_table, new_block_table, kv_lens, keep_lens, recent_lens, kept,
                dims):
    n, n_p, k, k_p = _pair(kv_lens, keep_lens, "kv_lens", "keep_lens")
    r, r_p = _per_task(recent_lens, "recent_lens", int(n.size))
    _mass_pool(mass, num_pages, dims)
    _block_table(block_table, int(n.size))
    new, new_p, stride = new_block_table, None, 0
    if new is not None:
        stride = _block_table(new, int(n.size))
        new_p = _dev(new, torch.int32, "new_block_table")
    total = _lens_total(k)
    if kept is not None and total is not None and kept.shape != (total, dims.num_kv_heads):
        raise ValueError("kept must have shape (%d, %d), got %s"
                         % (total, dims.num_kv_heads, tuple(kept.shape)))
    return (n, k, r), n_p, k_p, r_p, new_p, int(stride)


def tide_kv_evict(k_pool, v_pool, mass, block_table, kv_lens, keep_lens, dims: tide_dims,
                  recent_lens=None, new_block_table=None, kept=None, workspace=None,
                  stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    hold, n_p, k_p, r_p, new_p, stride = _evict_lens(mass, num_pages, block_table, new_block_table,
                                                     kv_lens, keep_lens, recent_lens, kept, dims)
    _same_device(k_pool, v_pool, mass, block_table, new_block_table, kept, workspace)
    ws, ws_n = _ws(workspace)
    _invoke("tide_kv_evict", k_pool, stream,
            _dev(k_pool, torch.bfloat16, "k_pool"), _dev(v_pool, torch.bfloat16, "v_pool"),
            _dev(mass, torch.float32, "mass"), num_pages,
            _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), new_p, stride,
            int(hold[0].size), n_p, k_p, r_p, ctypes.byref(dims),
            _dev(kept, torch.int32, "kept", nullable=True), ws, ws_n)


def tide_kv4_evict(kv4_pool, mass, block_table, kv_lens, keep_lens, dims: tide_dims,
                   recent_lens=None, new_block_table=None, kept=None, workspace=None,
                   stream=None) -> None:
    num_pages = _pool4_shape(kv4_pool, dims)
    hold, n_p, k_p, r_p, new_p, stride = _evict_lens(mass, num_pages, block_table, new_block_table,
                                                     kv_lens, keep_lens, recent_lens, kept, dims)
    _same_device(kv4_pool, mass, block_table, new_block_table, kept, workspace)
    ws, ws_n = _ws(workspace)
    _invoke("tide_kv4_evict", kv4_pool, stream,
            _dev(kv4_pool, torch.uint8, "kv4_pool"), _dev(mass, torch.float32, "mass"), num_pages,
            _dev(block_table, torch.int32, "block_table"), int(block_table.shape[1]), new_p, stride,
            int(hold[0].size), n_p, k_p, r_p, ctypes.byref(dims),
            _dev(kept, torch.int32, "kept", nullable=True), ws, ws_n)


# ---- steps whose rows, lengths and block lists are device data -------------------------------------
def _rows_workspace(name, op, num_rows, dims, budget, max_len):
    out = ctypes.c_size_t(0)
    _check(getattr(load(), name)(op, int(num_rows), int(budget), int(max_len), ctypes.byref(dims), ctypes.byref(out)),
           name)
    return int(out.value)


def tide_rows_workspace_size(op: int, num_rows: int, dims: tide_dims, budget: int = 0, max_len: int = 0) -> int:
    return _rows_workspace("tide_rows_workspace_size", op, num_rows, dims, budget, max_len)


def tide_rows_workspace_bound(op: int, num_rows: int, dims: tide_dims, budget: int = 0, max_len: int = 0) -> int:
    """Enough for every call with at most these rows, this budget and this longest context."""
    return _rows_workspace("tide_rows_workspace_bound", op, num_rows, dims, budget, max_len)


# A step of these calls is a few microseconds of GPU time, so what passes is checked in one look at each tensor.
_BF16, _I8, _I32T, _I64T, _F32 = torch.bfloat16, torch.int8, torch.int32, torch.int64, torch.float32


def _ptr(t, dtype, dev, name):
    """The address of a contiguous tensor of this type on device `dev`; else the error that says why not."""
    if isinstance(t, torch.Tensor):
        if t.dtype is dtype and t.get_device() == dev and dev >= 0 and t.is_contiguous():
            return t.data_ptr()
        if dev >= 0 and t.get_device() >= 0 and t.get_device() != dev:
            raise ValueError("all tensors of a call must be on one device, got %s for %s" % (t.device, name))
    return _dev(t, dtype, name)


def _vector(t, name, n):
    """t must be a 1-D tensor of n entries."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.shape != (n,):
        raise ValueError("%s must have shape (%d,), got %s" % (name, n, tuple(t.shape)))


def _count_of(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 1:
        raise ValueError("%s must be a 1-D tensor" % name)
    return t.shape[0]


def _bounds_pools(bounds, units, num_pages, dims):
    heads, d = dims.num_kv_heads, dims.head_dim
    if bounds.shape != (num_pages, heads, 2, d):
        raise ValueError("bounds must have shape %s, got %s" % ((num_pages, heads, 2, d), tuple(bounds.shape)))
    if units.shape != (num_pages, heads):
        raise ValueError("units must have shape %s, got %s" % ((num_pages, heads), tuple(units.shape)))


def tide_page_map(lens, want_lens, block_table, free_pages, free_count, lens_out, free_count_out, row_start,
                  row_task, row_pos, row_slot, dims: tide_dims, stream=None) -> None:
    """All of them device tensors: int32, row_slot int64."""
    n, rows = _count_of(lens, "lens"), _count_of(row_task, "row_task")
    _vector(want_lens, "want_lens", n)
    _vector(lens_out, "lens_out", n)
    _vector(free_count, "free_count", 1)
    _vector(free_count_out, "free_count_out", 1)
    _vector(row_start, "row_start", n + 1)
    _vector(row_pos, "row_pos", rows)
    _vector(row_slot, "row_slot", rows)
    stride = _block_table(block_table, n)
    capacity = _count_of(free_pages, "free_pages")
    dev = lens.get_device()
    _invoke("tide_page_map", lens, stream,
            _ptr(lens, _I32T, dev, "lens"), _ptr(want_lens, _I32T, dev, "want_lens"), n,
            _ptr(block_table, _I32T, dev, "block_table"), stride, _ptr(free_pages, _I32T, dev, "free_pages"), capacity,
            _ptr(free_count, _I32T, dev, "free_count"), rows, _ptr(lens_out, _I32T, dev, "lens_out"),
            _ptr(free_count_out, _I32T, dev, "free_count_out"), _ptr(row_start, _I32T, dev, "row_start"),
            _ptr(row_task, _I32T, dev, "row_task"), _ptr(row_pos, _I32T, dev, "row_pos"),
            _ptr(row_slot, _I64T, dev, "row_slot"), ctypes.byref(dims))


def tide_slot_append(k_new, v_new, row_slot, k_pool, v_pool, dims: tide_dims, bounds=None, units=None,
                     workspace=None, stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    rows = _count_of(row_slot, "row_slot")
    _rows(k_new, "k_new", rows, dims.num_kv_heads, dims.head_dim)
    _rows(v_new, "v_new", rows, dims.num_kv_heads, dims.head_dim)
    if (bounds is None) != (units is None):
        raise ValueError("bounds and units go together")
    dev, b, u = k_pool.get_device(), None, None
    if bounds is not None:
        _bounds_pools(bounds, units, num_pages, dims)
        b, u = _ptr(bounds, _I8, dev, "bounds"), _ptr(units, _I8, dev, "units")
    ws, ws_n = _ws(workspace)
    _same_device(k_pool, workspace)
    _invoke("tide_slot_append", k_pool, stream,
            _ptr(k_new, _BF16, dev, "k_new"), _ptr(v_new, _BF16, dev, "v_new"), _ptr(row_slot, _I64T, dev, "row_slot"),
            rows, _ptr(k_pool, _BF16, dev, "k_pool"), _ptr(v_pool, _BF16, dev, "v_pool"), num_pages, b, u,
            ctypes.byref(dims), ws, ws_n)


def tide_key_bounds(k_pool, block_table, lens, bounds, units, dims: tide_dims, from_lens=None, max_len: int = 0,
                    workspace=None, stream=None) -> None:
    num_pages = _pool_shape(k_pool, k_pool, dims)
    n = _count_of(lens, "lens")
    dev, start = k_pool.get_device(), None
    if from_lens is not None:
        _vector(from_lens, "from_lens", n)
        start = _ptr(from_lens, _I32T, dev, "from_lens")
    _bounds_pools(bounds, units, num_pages, dims)
    stride = _block_table(block_table, n)
    ws, ws_n = _ws(workspace)
    _same_device(k_pool, workspace)
    _invoke("tide_key_bounds", k_pool, stream,
            _ptr(k_pool, _BF16, dev, "k_pool"), num_pages, _ptr(block_table, _I32T, dev, "block_table"), stride, n,
            _ptr(lens, _I32T, dev, "lens"), start, int(max_len), _ptr(bounds, _I8, dev, "bounds"),
            _ptr(units, _I8, dev, "units"), ctypes.byref(dims), ws, ws_n)


def tide_block_select(q, row_task, row_pos, bounds, units, block_table, budget: int, dims: tide_dims, sel,
                      sink: int = 0, recent: int = 0, max_len: int = 0, workspace=None, stream=None) -> None:
    rows = _count_of(row_task, "row_task")
    _vector(row_pos, "row_pos", rows)
    _rows(q, "q", rows, dims.num_q_heads, dims.head_dim)
    num_pages = bounds.shape[0]
    _bounds_pools(bounds, units, num_pages, dims)
    if sel.shape != (rows, dims.num_kv_heads, budget):
        raise ValueError("sel must have shape (%d, %d, %d), got %s"
                         % (rows, dims.num_kv_heads, budget, tuple(sel.shape)))
    stride = _block_table(block_table, 0)
    dev = q.get_device()
    ws, ws_n = _ws(workspace)
    _same_device(q, workspace)
    _invoke("tide_block_select", q, stream,
            _ptr(q, _BF16, dev, "q"), _ptr(row_task, _I32T, dev, "row_task"), _ptr(row_pos, _I32T, dev, "row_pos"),
            rows, _ptr(bounds, _I8, dev, "bounds"), _ptr(units, _I8, dev, "units"), num_pages,
            _ptr(block_table, _I32T, dev, "block_table"), stride, block_table.shape[0], int(budget), int(sink),
            int(recent), int(max_len),
            ctypes.byref(dims), _ptr(sel, _I32T, dev, "sel"), ws, ws_n)


def tide_sparse_attn(q, k_pool, v_pool, block_table, row_task, row_pos, sel, dims: tide_dims, out, lse=None,
                     workspace=None, stream=None) -> None:
    num_pages = _pool_shape(k_pool, v_pool, dims)
    rows = _count_of(row_task, "row_task")
    _vector(row_pos, "row_pos", rows)
    _rows(q, "q", rows, dims.num_q_heads, dims.head_dim)
    _rows(out, "out", rows, dims.num_q_heads, dims.head_dim)
    _lse(lse, rows, dims.num_q_heads)
    if sel.dim() != 3 or sel.shape[0] != rows or sel.shape[1] != dims.num_kv_heads:
        raise ValueError("sel must be [%d][%d][budget], got %s" % (rows, dims.num_kv_heads, tuple(sel.shape)))
    stride = _block_table(block_table, 0)
    dev = k_pool.get_device()
    ws, ws_n = _ws(workspace)
    _same_device(k_pool, workspace)
    _invoke("tide_sparse_attn", k_pool, stream,
            _ptr(q, _BF16, dev, "q"), _ptr(k_pool, _BF16, dev, "k_pool"), _ptr(v_pool, _BF16, dev, "v_pool"), num_pages,
            _ptr(block_table, _I32T, dev, "block_table"), stride, block_table.shape[0],
            _ptr(row_task, _I32T, dev, "row_task"), _ptr(row_pos, _I32T, dev, "row_pos"), rows,
            _ptr(sel, _I32T, dev, "sel"), sel.shape[2], ctypes.byref(dims), _ptr(out, _BF16, dev, "out"),
            None if lse is None else _ptr(lse, _F32, dev, "lse"), ws, ws_n)


def tide_shutdown() -> None:
    load().tide_shutdown()
