"""ctypes binding of the C ABI in ``include/libra.h``.

Argument marshalling only: every step of the SpMM / SDDMM path runs inside
``liblibra.so``.  The module-level functions carry the same names as the C
entry points; :class:`Plan` bundles a plan handle with the device buffer that
backs it.  There is no fallback: if the shared library is missing, loading
raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# LIBRA_LIBRARY selects another build of the same library (e.g. an experimental one); default: the in-tree build
LIB_PATH = os.environ.get("LIBRA_LIBRARY") or os.path.join(_HERE, "liblibra.so")

F16, BF16, F32 = 0, 1, 2
MODE_HYBRID, MODE_DENSE_ONLY, MODE_SCALAR_ONLY = 0, 1, 2
FLAG_NO_FILL_PADDING, FLAG_NO_SPMM, FLAG_NO_SDDMM, FLAG_NATURAL_ORDER, FLAG_XCD_ORDER, FLAG_NO_XCD_ORDER = 1, 2, 4, 8, 16, 32
FLAG_SEGMENTS_BY_COLUMN, FLAG_TWO_KERNELS, FLAG_SEGMENTS_BY_COST = 64, 128, 256
TASK_WINDOW, TASK_CHUNK = 0, 1
OP_SPMM, OP_SDDMM = 1, 2
OK = 0
ERR = dict(NULL=-1, SHAPE=-2, ROWPTR=-3, COLUMN=-4, UNSORTED=-5, TOO_LARGE=-6, DTYPE=-7, OPTION=-8,
           UNSUPPORTED=-9, NOT_UPLOADED=-10, BUFFER=-11, NOT_BUILT=-12, HIP=-13, NOMEM=-14)


class LibraError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {strerror(code)} ({code})")


class PlanOpts(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("mode", C.c_int32), ("window_rows", C.c_int32),
                ("block_cols", C.c_int32), ("spmm_min_vec_nnz", C.c_int32), ("sddmm_min_blk_nnz", C.c_int32),
                ("ts", C.c_int32), ("cs", C.c_int32), ("short_len", C.c_int32), ("sddmm_cs", C.c_int32),
                ("flags", C.c_uint32), ("threads", C.c_int32), ("sddmm_ts", C.c_int32), ("sddmm_min_dense_pct", C.c_int32)]

    def __init__(self, **kw):
        super().__init__(**kw)
        self.struct_size = C.sizeof(PlanOpts)


INDEX_I32, INDEX_I64 = 0, 1
LOG_PROBS_MAX_TOP = 64
ADAMW_BLOCK = 256


class AdamwTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("first", C.c_void_p), ("second", C.c_void_p),
                ("first_scales", C.c_void_p), ("second_scales", C.c_void_p), ("master", C.c_void_p), ("n", C.c_int64),
                ("dtype", C.c_int32), ("number", C.c_uint32)]


class AdamwOpts(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("state_bits", C.c_int32), ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double),
                ("eps", C.c_double), ("weight_decay", C.c_double), ("step", C.c_int64), ("step_dev", C.c_void_p), ("lr_dev", C.c_void_p),
                ("seed", C.c_uint32)]

    def __init__(self, **kw):
        super().__init__(**kw)
        self.struct_size = C.sizeof(AdamwOpts)


class Task(C.Structure):
    _fields_ = [("kind", C.c_int32), ("id", C.c_int32), ("blk_begin", C.c_int32), ("blk_end", C.c_int32),
                ("res_begin", C.c_int32), ("res_end", C.c_int32),
                ("scalar_mask", C.c_uint32), ("atomic_mask", C.c_uint32), ("store_mask", C.c_uint32),
                ("cost", C.c_uint32)]


TASK_DTYPE = np.dtype([("kind", "<i4"), ("id", "<i4"), ("blk_begin", "<i4"), ("blk_end", "<i4"),
                       ("res_begin", "<i4"), ("res_end", "<i4"),
                       ("scalar_mask", "<u4"), ("atomic_mask", "<u4"), ("store_mask", "<u4"), ("cost", "<u4")])


class SubplanView(C.Structure):
    _fields_ = [("n_windows", C.c_int64), ("n_blocks", C.c_int64), ("n_dense_nnz", C.c_int64),
                ("n_res_nnz", C.c_int64), ("n_tasks", C.c_int64), ("n_zero_rows", C.c_int64),
                ("window_rows", C.c_int32), ("block_cols", C.c_int32), ("words_per_block", C.c_int32),
                ("value_dtype", C.c_int32),
                ("win_blkptr", C.c_void_p), ("blk_cols", C.c_void_p), ("blk_bitmap", C.c_void_p),
                ("blk_valptr", C.c_void_p), ("dense_val", C.c_void_p), ("dense_perm", C.c_void_p),
                ("win_resptr", C.c_void_p), ("res_row", C.c_void_p), ("res_col", C.c_void_p),
                ("res_val", C.c_void_p), ("res_perm", C.c_void_p), ("tasks", C.c_void_p),
                ("zero_rows", C.c_void_p)]


_STATS_I64 = ["M", "Kc", "nnz", "n_windows", "n_vectors", "n_vectors_nnz1",
              "spmm_dense_vectors", "spmm_blocks", "spmm_pad_slots", "spmm_dense_nnz", "spmm_res_nnz",
              "spmm_tasks", "spmm_chunk_tasks", "spmm_zero_rows",
              "spmm_short_rows", "spmm_long_rows", "spmm_split_rows", "spmm_gather_rows",
              "sddmm_dense_vectors", "sddmm_blocks", "sddmm_pad_slots", "sddmm_dense_nnz", "sddmm_res_nnz",
              "sddmm_tasks", "sddmm_gather_rows"]


class Stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in _STATS_I64] + [("plan_seconds", C.c_double), ("neighbour_share", C.c_double),
                                                               ("xcd_order", C.c_int64), ("device_seconds", C.c_double)]


_lib = None


def lib() -> C.CDLL:
    """Load liblibra.so (built by ``paper_2506_22714_amd.build``).  Raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2506_22714_amd.build` "
                               "(or __graft_entry__.build()) first")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        L.libra_plan.argtypes = [i64, i64, vp, vp, vp, C.c_int, C.POINTER(PlanOpts), C.POINTER(vp)]
        L.libra_plan_device_workspace.argtypes = [i64, i64, C.POINTER(PlanOpts), C.POINTER(sz)]
        L.libra_plan_device_buffer_bound.argtypes = [i64, i64, C.c_int, C.POINTER(PlanOpts), C.POINTER(sz)]
        L.libra_plan_device.argtypes = [i64, i64, i64, vp, vp, vp, C.c_int, C.POINTER(PlanOpts), vp, sz, vp, sz, C.c_int,
                                        vp, C.POINTER(vp)]
        L.libra_plan_device_bytes.argtypes = [vp, C.POINTER(sz)]
        L.libra_plan_upload.argtypes = [vp, vp, sz, vp]
        L.libra_spmm.argtypes = [vp, vp, i32, i64, vp, i64, vp]
        L.libra_spmm_rounded.argtypes = [vp, vp, i32, i64, vp, i64, vp, i64, vp]
        L.libra_sddmm.argtypes = [vp, vp, vp, i32, vp, vp]
        L.libra_sddmm_pattern.argtypes = [vp, vp, vp, i32, vp, vp]
        L.libra_edge_softmax.argtypes = [vp, vp, C.c_float, vp, C.c_int, vp]
        L.libra_edge_softmax_backward.argtypes = [vp, vp, C.c_int, vp, C.c_float, vp, vp]
        L.libra_sddmm_pattern_rounded.argtypes = [vp, vp, vp, i32, vp, vp]
        L.libra_edge_softmax_backward_rounded.argtypes = [vp, vp, vp, C.c_int, C.c_float, vp, vp]
        L.libra_value_products.argtypes = [vp, vp, i64, C.c_int, vp, vp]
        L.libra_embedding.argtypes = [vp, i64, i32, i64, C.c_int, vp, C.c_int, i64, C.c_float, vp, i64, vp]
        L.libra_embedding_backward_workspace.argtypes = [i64, i64, i32, C.POINTER(sz)]
        L.libra_embedding_backward.argtypes = [vp, i64, C.c_int, vp, C.c_int, i64, i64, i32, C.c_float, vp, i64, vp, sz, vp]
        L.libra_log_probs_workspace.argtypes = [i64, i64, i32, C.POINTER(sz)]
        L.libra_log_probs.argtypes = [vp, i64, i64, i64, C.c_int, vp, C.c_int, i32, C.c_float, vp, vp, vp, vp, vp, vp, sz, vp]
        L.libra_log_probs_backward.argtypes = [vp, i64, i64, i64, C.c_int, vp, C.c_int, i32, C.c_float, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.libra_adamw.argtypes = [vp, i32, C.POINTER(AdamwOpts), vp]
        L.libra_probe_coissue.argtypes = [C.c_int, vp, C.POINTER(C.c_float * 3), vp]
        L.libra_probe_gather.argtypes = [vp, i64, i32, vp, i64, vp, vp]
        L.libra_probe_gather_hub.argtypes = [vp, i64, i32, vp, i64, vp, i32, vp, vp]
        L.libra_csr_transpose_workspace.argtypes = [i64, C.POINTER(sz)]
        L.libra_csr_transpose_device.argtypes = [i64, i64, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        L.libra_csr_transpose_device_static.argtypes = [i64, i64, i64, vp, vp, vp, vp, vp, vp]
        L.libra_plan_set_values.argtypes = [vp, vp, C.c_int, vp]
        L.libra_plan_set_values_for.argtypes = [vp, vp, C.c_int, C.c_int, vp]
        L.libra_value_order_bytes.argtypes = [vp, C.POINTER(sz), C.POINTER(sz), C.POINTER(sz)]
        L.libra_value_order.argtypes = [vp, vp, vp, sz, vp, sz, vp]
        L.libra_plan_set_values_ordered.argtypes = [vp, vp, C.c_int, vp, vp, vp]
        L.libra_plan_export.argtypes = [vp, C.c_int, C.POINTER(SubplanView)]
        L.libra_plan_stats.argtypes = [vp, C.POINTER(Stats)]
        L.libra_plan_destroy.argtypes = [vp]
        L.libra_plan_destroy.restype = None
        L.libra_strerror.argtypes = [C.c_int]
        L.libra_strerror.restype = C.c_char_p
        L.libra_version.restype = C.c_int
        for n in ("libra_plan", "libra_plan_device_bytes", "libra_plan_upload", "libra_spmm", "libra_sddmm",
                  "libra_edge_softmax", "libra_plan_set_values", "libra_plan_export", "libra_plan_stats"):
            getattr(L, n).restype = C.c_int
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().libra_strerror(code).decode()


def libra_version() -> int:
    return int(lib().libra_version())


def _np_ptr(a):
    return None if a is None else C.c_void_p(a.ctypes.data)


def _np_dtype_code(a: np.ndarray) -> int:
    if a.dtype == np.float16:
        return F16
    if a.dtype == np.float32:
        return F32
    raise TypeError(f"unsupported value dtype {a.dtype}")


def _check(rc: int, what: str):
    if rc != OK:
        raise LibraError(rc, what)


# ---- entry points, same names as the C ABI (raw pointers / numpy host arrays in, codes checked) ----
def libra_plan(M: int, Kc: int, rowptr: np.ndarray, col: np.ndarray, val: np.ndarray, opts: PlanOpts | None = None,
               val_dtype: int | None = None) -> C.c_void_p:
    rowptr = np.ascontiguousarray(rowptr, dtype=np.int32)
    col = np.ascontiguousarray(col, dtype=np.int32)
    val = np.ascontiguousarray(val)
    handle = C.c_void_p()
    rc = lib().libra_plan(M, Kc, _np_ptr(rowptr), _np_ptr(col), _np_ptr(val),
                          _np_dtype_code(val) if val_dtype is None else val_dtype,
                          C.byref(opts) if opts is not None else None, C.byref(handle))
    _check(rc, "libra_plan")
    return handle


def libra_plan_device_workspace(M: int, nnz: int, opts: PlanOpts | None = None) -> int:
    n = C.c_size_t()
    _check(lib().libra_plan_device_workspace(M, nnz, C.byref(opts) if opts is not None else None, C.byref(n)),
           "libra_plan_device_workspace")
    return int(n.value)


def libra_plan_device_buffer_bound(M: int, nnz: int, val_dtype: int, opts: PlanOpts | None = None) -> int:
    n = C.c_size_t()
    _check(lib().libra_plan_device_buffer_bound(M, nnz, val_dtype, C.byref(opts) if opts is not None else None, C.byref(n)),
           "libra_plan_device_buffer_bound")
    return int(n.value)


def libra_plan_device(M: int, Kc: int, nnz: int, rowptr_ptr: int, col_ptr: int, val_ptr: int, val_dtype: int,
                      opts: PlanOpts | None, ws_ptr: int, ws_bytes: int, plan_ptr: int = 0, plan_bytes: int = 0,
                      keep_host_copy: bool = True, stream: int = 0) -> C.c_void_p:
    handle = C.c_void_p()
    rc = lib().libra_plan_device(M, Kc, nnz, C.c_void_p(rowptr_ptr), C.c_void_p(col_ptr), C.c_void_p(val_ptr), val_dtype,
                                 C.byref(opts) if opts is not None else None, C.c_void_p(ws_ptr), ws_bytes,
                                 C.c_void_p(plan_ptr), plan_bytes, 1 if keep_host_copy else 0,
                                 C.c_void_p(stream), C.byref(handle))
    _check(rc, "libra_plan_device")
    return handle


def libra_plan_device_bytes(plan) -> int:
    n = C.c_size_t()
    _check(lib().libra_plan_device_bytes(plan, C.byref(n)), "libra_plan_device_bytes")
    return int(n.value)


def libra_plan_upload(plan, dev_ptr: int, nbytes: int, stream: int = 0):
    _check(lib().libra_plan_upload(plan, C.c_void_p(dev_ptr), nbytes, C.c_void_p(stream)), "libra_plan_upload")


def libra_spmm(plan, B_ptr: int, N: int, ldb: int, C_ptr: int, ldc: int, stream: int = 0):
    _check(lib().libra_spmm(plan, C.c_void_p(B_ptr), N, ldb, C.c_void_p(C_ptr), ldc, C.c_void_p(stream)), "libra_spmm")


def libra_spmm_rounded(plan, B_ptr: int, N: int, ldb: int, R_ptr: int, ldr: int, scratch_ptr: int, lds: int, stream: int = 0):
    _check(lib().libra_spmm_rounded(plan, C.c_void_p(B_ptr), N, ldb, C.c_void_p(R_ptr), ldr, C.c_void_p(scratch_ptr), lds, C.c_void_p(stream)),
           "libra_spmm_rounded")


def libra_sddmm(plan, X_ptr: int, Y_ptr: int, K: int, out_ptr: int, stream: int = 0):
    _check(lib().libra_sddmm(plan, C.c_void_p(X_ptr), C.c_void_p(Y_ptr), K, C.c_void_p(out_ptr), C.c_void_p(stream)),
           "libra_sddmm")


def libra_sddmm_pattern(plan, X_ptr: int, Y_ptr: int, K: int, out_ptr: int, stream: int = 0):
    _check(lib().libra_sddmm_pattern(plan, C.c_void_p(X_ptr), C.c_void_p(Y_ptr), K, C.c_void_p(out_ptr), C.c_void_p(stream)),
           "libra_sddmm_pattern")


def libra_edge_softmax_backward(plan, alpha_ptr: int, alpha_dtype: int, dalpha_ptr: int, scale: float, dscores_ptr: int,
                                stream: int = 0):
    _check(lib().libra_edge_softmax_backward(plan, C.c_void_p(alpha_ptr), alpha_dtype, C.c_void_p(dalpha_ptr), C.c_float(scale),
                                             C.c_void_p(dscores_ptr), C.c_void_p(stream)), "libra_edge_softmax_backward")


def libra_value_products(vals_ptr: int, factors_ptr: int, n: int, dtype: int, out_ptr: int, stream: int = 0):
    _check(lib().libra_value_products(C.c_void_p(vals_ptr), C.c_void_p(factors_ptr), n, dtype, C.c_void_p(out_ptr), C.c_void_p(stream)),
           "libra_value_products")


def libra_embedding(table_ptr: int, rows: int, width: int, ld_table: int, dtype: int, index_ptr: int, index_type: int, n: int, scale: float,
                    out_ptr: int, ld_out: int, stream: int = 0):
    _check(lib().libra_embedding(table_ptr, rows, width, ld_table, dtype, index_ptr, index_type, n, scale, out_ptr, ld_out, stream), "libra_embedding")


def libra_embedding_backward_workspace(n: int, rows: int, width: int) -> int:
    b = C.c_size_t()
    _check(lib().libra_embedding_backward_workspace(n, rows, width, C.byref(b)), "libra_embedding_backward_workspace")
    return int(b.value)


def libra_embedding_backward(dout_ptr: int, ld_dout: int, dtype: int, index_ptr: int, index_type: int, n: int, rows: int, width: int,
                             scale: float, dtable_ptr: int, ld_dtable: int, ws_ptr: int, ws_bytes: int, stream: int = 0):
    _check(lib().libra_embedding_backward(dout_ptr, ld_dout, dtype, index_ptr, index_type, n, rows, width, scale, dtable_ptr, ld_dtable,
                                          ws_ptr, ws_bytes, stream), "libra_embedding_backward")


def libra_log_probs_workspace(n: int, classes: int, top: int) -> int:
    b = C.c_size_t()
    _check(lib().libra_log_probs_workspace(n, classes, top, C.byref(b)), "libra_log_probs_workspace")
    return int(b.value)


def libra_log_probs(logits_ptr: int, n: int, classes: int, ld: int, dtype: int, targets_ptr: int, index_type: int, top: int, scale: float,
                    target_ptr: int, entropy_ptr: int, top_ptr: int, top_index_ptr: int, stats_ptr: int, ws_ptr: int = 0, ws_bytes: int = 0,
                    stream: int = 0):
    _check(lib().libra_log_probs(logits_ptr, n, classes, ld, dtype, targets_ptr, index_type, top, scale, target_ptr, entropy_ptr, top_ptr,
                                 top_index_ptr, stats_ptr, ws_ptr, ws_bytes, stream), "libra_log_probs")


def libra_log_probs_backward(logits_ptr: int, n: int, classes: int, ld: int, dtype: int, targets_ptr: int, index_type: int, top: int,
                             scale: float, entropy_ptr: int, stats_ptr: int, top_index_ptr: int, d_target_ptr: int, d_entropy_ptr: int,
                             d_top_ptr: int, dlogits_ptr: int, ld_dlogits: int, stream: int = 0):
    _check(lib().libra_log_probs_backward(logits_ptr, n, classes, ld, dtype, targets_ptr, index_type, top, scale, entropy_ptr, stats_ptr,
                                          top_index_ptr, d_target_ptr, d_entropy_ptr, d_top_ptr, dlogits_ptr, ld_dlogits, stream),
           "libra_log_probs_backward")


def libra_adamw(tensors, count: int, opts: AdamwOpts, stream: int = 0):
    """`tensors`: a ctypes array of :class:`AdamwTensor`."""
    _check(lib().libra_adamw(tensors, count, C.byref(opts), stream), "libra_adamw")


def libra_probe_coissue(iters: int, sink_ptr: int, stream: int = 0):
    """(MFMA only, FMA only, both) in microseconds."""
    t = (C.c_float * 3)()
    _check(lib().libra_probe_coissue(iters, C.c_void_p(sink_ptr), C.byref(t), C.c_void_p(stream)), "libra_probe_coissue")
    return tuple(float(x) for x in t)


def libra_probe_gather(table_ptr: int, table_rows: int, row_bytes: int, idx_ptr: int, n: int, sink_ptr: int, stream: int = 0):
    _check(lib().libra_probe_gather(C.c_void_p(table_ptr), table_rows, row_bytes, C.c_void_p(idx_ptr), n, C.c_void_p(sink_ptr),
                                    C.c_void_p(stream)), "libra_probe_gather")


def libra_probe_gather_hub(table_ptr: int, table_rows: int, row_bytes: int, idx_ptr: int, n: int, hub_rows_ptr: int, n_hub: int,
                           sink_ptr: int, stream: int = 0):
    _check(lib().libra_probe_gather_hub(C.c_void_p(table_ptr), table_rows, row_bytes, C.c_void_p(idx_ptr), n,
                                        C.c_void_p(hub_rows_ptr), n_hub, C.c_void_p(sink_ptr), C.c_void_p(stream)), "libra_probe_gather_hub")


def libra_csr_transpose_workspace(nnz: int) -> int:
    n = C.c_size_t()
    _check(lib().libra_csr_transpose_workspace(nnz, C.byref(n)), "libra_csr_transpose_workspace")
    return int(n.value)


def libra_csr_transpose_device(M: int, Kc: int, nnz: int, rowptr_ptr: int, col_ptr: int, rowptr_t_ptr: int, col_t_ptr: int,
                               perm_t_ptr: int, ws_ptr: int, ws_bytes: int, stream: int = 0):
    _check(lib().libra_csr_transpose_device(M, Kc, nnz, C.c_void_p(rowptr_ptr), C.c_void_p(col_ptr), C.c_void_p(rowptr_t_ptr),
                                            C.c_void_p(col_t_ptr), C.c_void_p(perm_t_ptr), C.c_void_p(ws_ptr), ws_bytes,
                                            C.c_void_p(stream)), "libra_csr_transpose_device")


TRANSPOSE_STATIC_MAX_NNZ = 1 << 20


def libra_csr_transpose_device_static(M: int, Kc: int, nnz: int, rowptr_ptr: int, col_ptr: int, rowptr_t_ptr: int, col_t_ptr: int,
                                      perm_t_ptr: int, stream: int = 0):
    _check(lib().libra_csr_transpose_device_static(M, Kc, nnz, C.c_void_p(rowptr_ptr), C.c_void_p(col_ptr), C.c_void_p(rowptr_t_ptr),
                                                   C.c_void_p(col_t_ptr), C.c_void_p(perm_t_ptr), C.c_void_p(stream)),
           "libra_csr_transpose_device_static")


def _csr_operands(M: int, rowptr, col) -> int:
    """Checks the device CSR arrays a planner or the transposition reads (sizes, types, layout, device); returns nnz."""
    import torch
    for name, t in (("rowptr", rowptr), ("col", col)):
        if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous int32 torch tensor")
    if rowptr.numel() != M + 1:
        raise ValueError(f"rowptr: {rowptr.numel()} elements, expected M + 1 = {M + 1}")
    if not rowptr.is_cuda or not col.is_cuda or col.device != rowptr.device:
        raise ValueError("rowptr and col must be on one GPU")
    return int(col.numel())


def transpose_csr(M: int, Kc: int, rowptr, col):
    """(rowptr_t, col_t, perm_t) of the transposed pattern, torch int32 tensors on the device of the inputs."""
    import torch
    nnz = int(col.numel())
    _csr_operands(M, rowptr, col)
    rowptr_t = torch.empty(Kc + 1, dtype=torch.int32, device=rowptr.device)
    col_t = torch.empty(nnz, dtype=torch.int32, device=rowptr.device)
    perm_t = torch.empty(nnz, dtype=torch.int32, device=rowptr.device)
    nb = libra_csr_transpose_workspace(nnz)
    ws = torch.empty(nb, dtype=torch.uint8, device=rowptr.device)
    libra_csr_transpose_device(M, Kc, nnz, rowptr.data_ptr(), col.data_ptr() if nnz else 0, rowptr_t.data_ptr(),
                               col_t.data_ptr() if nnz else 0, perm_t.data_ptr() if nnz else 0, ws.data_ptr(), nb,
                               torch.cuda.current_stream().cuda_stream)
    return rowptr_t, col_t, perm_t


def libra_edge_softmax(plan, scores_ptr: int, scale: float, out_ptr: int, out_dtype: int, stream: int = 0):
    _check(lib().libra_edge_softmax(plan, C.c_void_p(scores_ptr), C.c_float(scale), C.c_void_p(out_ptr), out_dtype,
                                    C.c_void_p(stream)), "libra_edge_softmax")


def libra_plan_set_values(plan, vals_ptr: int, dtype: int, stream: int = 0):
    _check(lib().libra_plan_set_values(plan, C.c_void_p(vals_ptr), dtype, C.c_void_p(stream)), "libra_plan_set_values")


def libra_plan_set_values_for(plan, vals_ptr: int, dtype: int, ops: int, stream: int = 0):
    _check(lib().libra_plan_set_values_for(plan, C.c_void_p(vals_ptr), dtype, ops, C.c_void_p(stream)),
           "libra_plan_set_values_for")


def libra_value_order_bytes(plan) -> tuple:
    """(order, workspace, scratch) in bytes."""
    n = [C.c_size_t() for _ in range(3)]
    _check(lib().libra_value_order_bytes(plan, *(C.byref(x) for x in n)), "libra_value_order_bytes")
    return tuple(int(x.value) for x in n)


def libra_value_order(plan, perm_ptr: int, order_ptr: int, order_bytes: int, ws_ptr: int, ws_bytes: int, stream: int = 0):
    _check(lib().libra_value_order(plan, C.c_void_p(perm_ptr), C.c_void_p(order_ptr), order_bytes, C.c_void_p(ws_ptr), ws_bytes,
                                   C.c_void_p(stream)), "libra_value_order")


def libra_plan_destroy(plan):
    lib().libra_plan_destroy(plan)


def _arr(ptr, n, dtype):
    if not ptr or n == 0:
        return np.zeros(0, dtype=dtype)
    buf = (C.c_char * (n * np.dtype(dtype).itemsize)).from_address(ptr)
    return np.frombuffer(buf, dtype=dtype).copy()


def libra_plan_export(plan, which: int) -> dict:
    """Copies of one sub-plan's host arrays as numpy arrays (0 = SpMM, 1 = SDDMM)."""
    v = SubplanView()
    _check(lib().libra_plan_export(plan, which, C.byref(v)), "libra_plan_export")
    vt = {F16: np.float16, BF16: np.uint16, F32: np.float32}[v.value_dtype]      # bfloat16 comes back as bit patterns
    nb, KB, wpb = v.n_blocks, v.block_cols, v.words_per_block
    out = dict(n_windows=v.n_windows, n_blocks=nb, n_dense_nnz=v.n_dense_nnz, n_res_nnz=v.n_res_nnz,
               n_tasks=v.n_tasks, window_rows=v.window_rows, block_cols=KB, words_per_block=wpb,
               win_blkptr=_arr(v.win_blkptr, v.n_windows + 1, np.int32),
               blk_cols=_arr(v.blk_cols, nb * KB, np.int32).reshape(nb, KB),
               blk_bitmap=_arr(v.blk_bitmap, nb * wpb, np.uint64).reshape(nb, wpb),
               blk_valptr=_arr(v.blk_valptr, nb + 1, np.int32),
               dense_val=_arr(v.dense_val, v.n_dense_nnz, vt),
               dense_perm=_arr(v.dense_perm, v.n_dense_nnz, np.int32),
               res_row=_arr(v.res_row, v.n_res_nnz, np.int32),
               res_col=_arr(v.res_col, v.n_res_nnz, np.int32),
               res_val=_arr(v.res_val, v.n_res_nnz, vt),
               res_perm=_arr(v.res_perm, v.n_res_nnz, np.int32),
               tasks=_arr(v.tasks, v.n_tasks, TASK_DTYPE),
               zero_rows=_arr(v.zero_rows, v.n_zero_rows, np.int32))
    if which == 0:
        out["win_resptr"] = _arr(v.win_resptr, v.n_windows + 1, np.int32)
    return out


def libra_plan_stats(plan) -> dict:
    s = Stats()
    _check(lib().libra_plan_stats(plan, C.byref(s)), "libra_plan_stats")
    return {n: getattr(s, n) for n, _t in Stats._fields_}


def _with_tuned(opts: dict, tuned, val_dtype: int, N, K) -> dict:
    """Plan options with the entries of a tuner table filled in (argument marshalling: the table is data, the choice was
    made by the tuner); options given explicitly (non-zero) are kept."""
    if tuned is None:
        return opts
    from .tune import tuned_options
    t = tuned_options(tuned, {F16: "f16", BF16: "bf16", F32: "f32"}[val_dtype], N=N, K=K)
    return {**t, **{k: v for k, v in opts.items() if v or k not in t}}


# ---- convenience wrapper: a plan handle plus the torch buffer that backs its device copy ----
# A call on a small matrix takes less time on the GPU than a handful of Python attribute chains: operands that are what they should be
# are recognised by one short test, and everything else goes through the checks that say what is wrong.
_torch = None


def _gpu():
    """torch, with the stream lookup that does not build a Stream object if this torch has it."""
    global _torch, _stream
    if _torch is None:
        import torch
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and device is not None:
            _stream = lambda: raw(device())                                         # noqa: E731
        _torch = torch
    return _torch


def _stream():
    return _gpu().cuda.current_stream().cuda_stream


def _is_matrix(t, dtype, rows: int) -> bool:
    return isinstance(t, _torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous() and t.dim() == 2 and t.shape[0] == rows


def _is_vector(t, dtype, n: int) -> bool:
    return isinstance(t, _torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous() and t.numel() == n


class ValueOrder(tuple):
    """(array, scratch bytes) of :meth:`Plan.value_order`, with the plan that it was made for."""
    plan = None


class Plan:
    def __init__(self, M, Kc, rowptr, col, val, val_dtype: int | None = None, tuned=None, N: int | None = None,
                 K: int | None = None, **opts):
        """`val_dtype=BF16` with `val` as uint16 bit patterns builds a bfloat16 plan (numpy has no such type).
        `tuned`: a table written by `python -m paper_2506_22714_amd.tune --emit` (path or dict); the options of the
        classes of the feature widths `N` (SpMM) and `K` (SDDMM) are taken from it, explicit options win."""
        self.M, self.Kc = int(M), int(Kc)
        self.val_dtype = _np_dtype_code(np.asarray(val)) if val_dtype is None else int(val_dtype)
        opts = _with_tuned(opts, tuned, self.val_dtype, N, K)
        self.handle = libra_plan(self.M, self.Kc, rowptr, col, val, PlanOpts(**opts) if opts else None,
                                 val_dtype=self.val_dtype)
        self._facts(opts)
        self._buf = None

    @classmethod
    def from_device_csr(cls, M, Kc, rowptr, col, val, resident: bool = False, keep_host_copy: bool = True, tuned=None,
                        N: int | None = None, K: int | None = None, **opts):
        """Plan built on the GPU from torch tensors (int32 rowptr/col, float16 / bfloat16 / float32 values).
        ``resident``: the device copy is written during planning into a buffer of the bound size (no upload).
        ``tuned``, ``N``, ``K``: as in the constructor."""
        import torch
        nnz = _csr_operands(M, rowptr, col)
        if val.dtype not in (torch.float16, torch.bfloat16, torch.float32):
            raise ValueError(f"val: dtype {val.dtype} is not float16, bfloat16 or float32")
        if val.numel() != nnz or not val.is_contiguous():
            raise ValueError(f"val: {val.numel()} elements (contiguous: {val.is_contiguous()}), expected {nnz} contiguous")
        if not val.is_cuda or val.device != rowptr.device:
            raise ValueError("val: must be on the same GPU as rowptr")
        self = cls.__new__(cls)
        self.M, self.Kc = int(M), int(Kc)
        self.val_dtype = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}[val.dtype]
        opts = _with_tuned(opts, tuned, self.val_dtype, N, K)
        o = PlanOpts(**opts) if opts else None
        ws_bytes = libra_plan_device_workspace(self.M, nnz, o)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=rowptr.device)
        self.handle = None
        self._buf = None
        if resident:
            nb = libra_plan_device_buffer_bound(self.M, nnz, self.val_dtype, o)
            self._buf = torch.empty(nb, dtype=torch.uint8, device=rowptr.device)
        self.handle = libra_plan_device(self.M, self.Kc, nnz, rowptr.data_ptr(), col.data_ptr() if nnz else 0,
                                        val.data_ptr() if nnz else 0, self.val_dtype, o, ws.data_ptr(), ws_bytes,
                                        self._buf.data_ptr() if resident else 0, self._buf.numel() if resident else 0,
                                        keep_host_copy or not resident, torch.cuda.current_stream().cuda_stream)
        del ws
        self._facts(opts)
        return self

    _dtype_cached = None

    def _facts(self, opts):
        self._lib = lib()
        self._token = object()              # what the orders of this plan's values carry
        stats = libra_plan_stats(self.handle)
        self.nnz = stats["nnz"]
        # rows that a call with rounded results sums up in fp32 memory: those with several writers, all of them in two-kernel mode
        self._fp32_rows = stats["spmm_zero_rows"] > 0 or bool(opts.get("flags", 0) & FLAG_TWO_KERNELS)

    @classmethod
    def from_csr(cls, csr, val=None, val_dtype: int | None = None, tuned=None, N: int | None = None, K: int | None = None, **opts):
        return cls(csr.M, csr.Kc, csr.rowptr, csr.col, csr.val if val is None else val, val_dtype=val_dtype, tuned=tuned, N=N, K=K, **opts)

    def close(self):
        if self.handle is not None:
            libra_plan_destroy(self.handle)
            self.handle = None
            self._buf = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def stats(self) -> dict:
        return libra_plan_stats(self.handle)

    def export(self, which: int) -> dict:
        return libra_plan_export(self.handle, which)

    def upload(self, device="cuda"):
        import torch
        n = libra_plan_device_bytes(self.handle)
        self._buf = torch.empty(n, dtype=torch.uint8, device=device)
        libra_plan_upload(self.handle, self._buf.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
        return self

    @property
    def _dtype(self):
        d = self._dtype_cached
        if d is None:
            torch = _gpu()
            d = self._dtype_cached = {F16: torch.float16, BF16: torch.bfloat16, F32: torch.float32}[self.val_dtype]
        return d

    # The C ABI sees pointers only: the sizes behind them are checked here, before any launch, and a mismatch raises
    # (an undersized operand would make a kernel read or write past its end).  Shape, type and layout first, the device last.
    @staticmethod
    def _operand(t, name, dtype, shape=None, numel=None, rows_contiguous=False):
        import torch
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name}: expected a torch tensor, got {type(t).__name__}")
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
        if shape is not None:
            if t.dim() != len(shape) or any(want is not None and int(have) != int(want) for have, want in zip(t.shape, shape)):
                raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple('*' if w is None else w for w in shape)}")
        if numel is not None and t.numel() != numel:
            raise ValueError(f"{name}: {t.numel()} elements, expected {numel}")
        if rows_contiguous:
            if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
                raise ValueError(f"{name}: rows must be contiguous (strides {tuple(t.stride())})")
        elif not t.is_contiguous():
            raise ValueError(f"{name}: must be contiguous")
        if not t.is_cuda:
            raise ValueError(f"{name}: must be a GPU tensor")

    def _value_code(self, t, name):
        import torch
        code = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}.get(t.dtype)
        if code is None:
            raise ValueError(f"{name}: dtype {t.dtype} is not float16, bfloat16 or float32")
        return code

    def _check_matrix(self, t, name, rows, cols=None, rows_contiguous=False):
        if not (_is_matrix(t, self._dtype, rows) and (cols is None or t.shape[1] == cols)):
            self._operand(t, name, self._dtype, shape=(rows, cols), rows_contiguous=rows_contiguous)

    def _check_vector(self, t, name, dtype):
        if not _is_vector(t, dtype, self.nnz):
            self._operand(t, name, dtype, numel=self.nnz)

    def spmm(self, B, out=None):
        torch = _gpu()
        self._check_matrix(B, "B", self.Kc, rows_contiguous=True)
        N = B.shape[1]
        if out is None:
            out = torch.empty((self.M, N), dtype=torch.float32, device=B.device)
        else:
            if not (_is_matrix(out, torch.float32, self.M) and out.shape[1] == N):
                self._operand(out, "out", torch.float32, shape=(self.M, N), rows_contiguous=True)
            if out.get_device() != B.get_device():
                raise ValueError("out: on another device than B")
        rc = self._lib.libra_spmm(self.handle, B.data_ptr(), N, B.stride(0), out.data_ptr(), out.stride(0), _stream())
        if rc:
            _check(rc, "libra_spmm")
        return out

    def spmm_rounded(self, B):
        """``spmm(B)`` in the plan's value type: the fp32 sums rounded once."""
        if self.val_dtype == F32:
            return self.spmm(B)
        torch = _gpu()
        self._check_matrix(B, "B", self.Kc, rows_contiguous=True)
        N = B.shape[1]
        out = torch.empty((self.M, N), dtype=B.dtype, device=B.device)
        scratch = torch.empty((self.M, N), dtype=torch.float32, device=B.device) if self._fp32_rows else None
        rc = self._lib.libra_spmm_rounded(self.handle, B.data_ptr(), N, B.stride(0), out.data_ptr(), N, scratch.data_ptr() if scratch is not None else 0, N,
                                          _stream())
        if rc:
            _check(rc, "libra_spmm_rounded")
        return out

    def sddmm(self, X, Y, out=None, pattern_only: bool = False):
        torch = _gpu()
        self._check_matrix(X, "X", self.M)
        K = X.shape[1]
        self._check_matrix(Y, "Y", self.Kc, K)
        if out is None:
            out = torch.empty(self.nnz, dtype=torch.float32, device=X.device)
        else:
            self._check_vector(out, "out", torch.float32)
        if not X.get_device() == Y.get_device() == out.get_device():
            raise ValueError("X, Y and out must be on one device")
        call = self._lib.libra_sddmm_pattern if pattern_only else self._lib.libra_sddmm
        rc = call(self.handle, X.data_ptr(), Y.data_ptr(), K, out.data_ptr(), _stream())
        if rc:
            _check(rc, "libra_sddmm_pattern" if pattern_only else "libra_sddmm")
        return out

    def sddmm_pattern_rounded(self, X, Y):
        """``sddmm(X, Y, pattern_only=True)`` in the plan's value type, rounded once."""
        if self.val_dtype == F32:
            return self.sddmm(X, Y, pattern_only=True)
        torch = _gpu()
        self._check_matrix(X, "X", self.M)
        K = X.shape[1]
        self._check_matrix(Y, "Y", self.Kc, K)
        if Y.get_device() != X.get_device():
            raise ValueError("X and Y must be on one device")
        out = torch.empty(self.nnz, dtype=X.dtype, device=X.device)
        rc = self._lib.libra_sddmm_pattern_rounded(self.handle, X.data_ptr(), Y.data_ptr(), K, out.data_ptr(), _stream())
        if rc:
            _check(rc, "libra_sddmm_pattern_rounded")
        return out

    def edge_softmax(self, scores, scale: float, out=None):
        torch = _gpu()
        self._check_vector(scores, "scores", torch.float32)
        if out is None:
            out, code = torch.empty(self.nnz, dtype=self._dtype, device=scores.device), self.val_dtype
        else:
            code = self._value_code(out, "out")
            self._check_vector(out, "out", out.dtype)
            if out.get_device() != scores.get_device():
                raise ValueError("out: on another device than scores")
        rc = self._lib.libra_edge_softmax(self.handle, scores.data_ptr(), scale, out.data_ptr(), code, _stream())
        if rc:
            _check(rc, "libra_edge_softmax")
        return out

    def edge_softmax_backward(self, alpha, dalpha, scale: float, out=None):
        torch = _gpu()
        code = self._value_code(alpha, "alpha")
        self._check_vector(alpha, "alpha", alpha.dtype)
        self._check_vector(dalpha, "dalpha", torch.float32)
        if out is None:
            out = torch.empty(self.nnz, dtype=torch.float32, device=alpha.device)
        else:
            self._check_vector(out, "out", torch.float32)
        if not alpha.get_device() == dalpha.get_device() == out.get_device():
            raise ValueError("alpha, dalpha and out must be on one device")
        rc = self._lib.libra_edge_softmax_backward(self.handle, alpha.data_ptr(), code, dalpha.data_ptr(), scale, out.data_ptr(), _stream())
        if rc:
            _check(rc, "libra_edge_softmax_backward")
        return out

    def edge_softmax_backward_rounded(self, alpha, dalpha, scale: float):
        """``edge_softmax_backward`` of a ``dalpha`` in alpha's type."""
        torch = _gpu()
        code = self._value_code(alpha, "alpha")
        self._check_vector(alpha, "alpha", alpha.dtype)
        self._check_vector(dalpha, "dalpha", alpha.dtype)
        if dalpha.get_device() != alpha.get_device():
            raise ValueError("alpha and dalpha must be on one device")
        out = torch.empty(self.nnz, dtype=torch.float32, device=alpha.device)
        rc = self._lib.libra_edge_softmax_backward_rounded(self.handle, alpha.data_ptr(), dalpha.data_ptr(), code, scale, out.data_ptr(), _stream())
        if rc:
            _check(rc, "libra_edge_softmax_backward_rounded")
        return out

    def value_products(self, vals, factors):
        """``(factors * vals.float())`` in the plan's value type, rounded once: values of A (CSR order) times fp32 factors."""
        if self.val_dtype == F32:
            return factors * vals
        torch = _gpu()
        self._check_vector(vals, "vals", self._dtype)
        self._check_vector(factors, "factors", torch.float32)
        if factors.get_device() != vals.get_device():
            raise ValueError("vals and factors must be on one device")
        out = torch.empty(self.nnz, dtype=vals.dtype, device=vals.device)
        rc = self._lib.libra_value_products(vals.data_ptr(), factors.data_ptr(), self.nnz, self.val_dtype, out.data_ptr(), _stream())
        if rc:
            _check(rc, "libra_value_products")
        return out

    def set_values(self, vals, ops: int = OP_SPMM | OP_SDDMM, one_call: bool = False):
        """New values of A in CSR order.  ``one_call``: through libra_plan_set_values (both operators) instead of
        libra_plan_set_values_for."""
        _gpu()
        self._check_vector(vals, "vals", self._dtype)
        if one_call:
            if ops != OP_SPMM | OP_SDDMM:
                raise ValueError("one_call refreshes both operators")
            libra_plan_set_values(self.handle, vals.data_ptr(), self.val_dtype, _stream())
            return
        rc = self._lib.libra_plan_set_values_for(self.handle, vals.data_ptr(), self.val_dtype, ops, _stream())
        if rc:
            _check(rc, "libra_plan_set_values_for")

    def value_order(self, perm):
        """The form of a permutation of the nonzeros (int32) that :meth:`set_values_ordered` of this plan reads."""
        torch = _gpu()
        self._check_vector(perm, "perm", torch.int32)
        order_bytes, ws_bytes, scratch_bytes = libra_value_order_bytes(self.handle)
        order = torch.empty(order_bytes, dtype=torch.uint8, device=perm.device)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=perm.device)
        libra_value_order(self.handle, perm.data_ptr(), order.data_ptr(), order_bytes, ws.data_ptr(), ws_bytes, _stream())
        made = ValueOrder((order, scratch_bytes))
        made.plan = self._token
        return made

    def set_values_ordered(self, vals, order):
        """SpMM values from ``vals`` in the order that ``order`` (of :meth:`value_order`) stands for: nonzero p takes vals[perm[p]]."""
        torch = _gpu()
        self._check_vector(vals, "vals", self._dtype)
        if getattr(order, "plan", None) is not self._token:      # the kernels take its places and sizes as they are
            raise ValueError("order: not made by value_order of this plan")
        order, scratch_bytes = order
        if order.get_device() != vals.get_device():
            raise ValueError("vals: on another device than order")
        scratch = torch.empty(scratch_bytes, dtype=torch.uint8, device=vals.device) if scratch_bytes else None
        rc = self._lib.libra_plan_set_values_ordered(self.handle, vals.data_ptr(), self.val_dtype, order.data_ptr(),
                                                     scratch.data_ptr() if scratch is not None else 0, _stream())
        if rc:
            _check(rc, "libra_plan_set_values_ordered")


# ---- the ends of a training step: no plan, any GPU (the call is made on the device and the current stream of its operands) ----
def _launch(call, what: str, like, *args):
    """call(*args, stream) on the device of the tensor `like`."""
    cuda = _torch.cuda
    if like.get_device() == cuda.current_device():
        rc = call(*args, _stream())
    else:
        with cuda.device(like.device):
            rc = call(*args, cuda.current_stream().cuda_stream)
    if rc:
        _check(rc, what)


def _code(t, name: str) -> int:
    torch = _torch
    d = t.dtype if isinstance(t, torch.Tensor) else None
    if d is torch.float16:
        return F16
    if d is torch.bfloat16:
        return BF16
    if d is torch.float32:
        return F32
    raise ValueError(f"{name}: expected a torch tensor of float16, bfloat16 or float32, got {d or type(t).__name__}")


def _rows_of(t, name: str, cols=None, like=None) -> int:
    """A matrix whose rows are contiguous (with any distance between them); its type's code."""
    code = _code(t, name)
    shape = t.shape
    if len(shape) != 2 or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name}: shape {tuple(shape)}, expected ('*', {'*' if cols is None else cols})")
    if not t.is_contiguous() and (shape[1] > 1 and t.stride(1) != 1 or shape[0] > 1 and t.stride(0) < shape[1]):
        raise ValueError(f"{name}: rows must be contiguous (strides {tuple(t.stride())})")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a GPU tensor")
    if like is not None and (t.get_device() != like.get_device() or t.dtype is not like.dtype):
        raise ValueError(f"{name}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    return code


def _width(t, name: str) -> int:
    """Elements of a row, which the library counts in 32 bits."""
    width = t.shape[1]
    if not 1 <= width < 1 << 31:
        raise ValueError(f"{name}: rows of {width or 'no'} elements")
    return width


def _ld(t) -> int:
    return t.shape[1] if t.is_contiguous() or t.shape[0] <= 1 else t.stride(0)


def _apart(out, t, name: str):
    """Refuses a result that lies on one of its inputs (columns of one array beside each other are fine)."""
    a, b, size, ld = out.data_ptr(), t.data_ptr(), t.element_size(), _ld(t)
    if out.numel() == 0 or t.numel() == 0:
        return
    if a >= b + ((t.shape[0] - 1) * ld + t.shape[1]) * size or b >= a + ((out.shape[0] - 1) * _ld(out) + out.shape[1]) * size:
        return
    lds = {_ld(x) for x in (out, t) if x.shape[0] > 1}       # (one row goes by the distance of the other's rows)
    if len(lds) == 1:
        (ld,) = lds
        column = (a - b) // size % ld
        if column >= t.shape[1] and column + out.shape[1] <= ld:
            return
    raise ValueError(f"out: overlaps {name}")


def _index_code(t, name: str, like) -> int:
    torch = _torch
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.int32, torch.int64) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous int32 or int64 torch tensor")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name}: must be a tensor on {like.device}")
    return INDEX_I64 if t.dtype is torch.int64 else INDEX_I32


def _fp32_on(t, name: str, shape, like):
    torch = _torch
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous float32 torch tensor of shape {tuple(shape)}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name}: must be a tensor on {like.device}")
    return t.data_ptr()


def embedding(table, index, scale: float = 1.0, out=None):
    """``scale * table[index]`` in the table's type, rounded once.  ``index`` (int32 or int64, any shape): -1 is padding, a row of zeros;
    another number outside the table gives a row of NaN.  ``out``: matrix of index.numel() rows to write to."""
    torch = _gpu()
    dtype = _rows_of(table, "table")
    kind = _index_code(index, "index", table)
    n, rows, width = index.numel(), table.shape[0], _width(table, "table")
    if out is None:
        out, ld_out = torch.empty(*index.shape, width, dtype=table.dtype, device=table.device), width
    else:
        _rows_of(out, "out", width, like=table)
        if out.shape[0] != n:
            raise ValueError(f"out: {out.shape[0]} rows, expected {n}")
        _apart(out, table, "table")
        ld_out = _ld(out)
    _launch(lib().libra_embedding, "libra_embedding", table, table.data_ptr(), rows, width, _ld(table), dtype, index.data_ptr(), kind, n, scale,
            out.data_ptr(), ld_out)
    return out


def embedding_backward(dout, index, rows: int, scale: float = 1.0, out=None):
    """Gradient of ``embedding(table, index, scale)`` with respect to a table of ``rows`` rows, from the gradient ``dout`` (a row per id)
    of its result: rows of equal ids are added in fp32, in an order that depends on the ids, the shapes and the type alone, and rounded once
    to dout's type."""
    torch = _gpu()
    dtype = _rows_of(dout, "dout")
    kind = _index_code(index, "index", dout)
    n, width = dout.shape[0], _width(dout, "dout")
    if index.numel() != n:
        raise ValueError(f"index: {index.numel()} ids for {n} rows of dout")
    nb = libra_embedding_backward_workspace(n, rows, width)
    if out is None:
        out = torch.empty(rows, width, dtype=dout.dtype, device=dout.device)
    else:
        _rows_of(out, "out", width, like=dout)
        if out.shape[0] != rows:
            raise ValueError(f"out: {out.shape[0]} rows, expected {rows}")
        _apart(out, dout, "dout")
    ws = torch.empty(nb, dtype=torch.uint8, device=dout.device)
    _launch(lib().libra_embedding_backward, "libra_embedding_backward", dout, dout.data_ptr(), _ld(dout), dtype, index.data_ptr(), kind, n, rows,
            width, scale, out.data_ptr(), _ld(out), ws.data_ptr(), nb)
    return out


class LogProbs(NamedTuple):
    """What :func:`log_probs` gives for n rows of logits: log probability of the given class (None without targets) and entropy, fp32[n];
    the ``top`` most likely classes, int64[n, top], and their log probabilities, fp32[n, top]; ``stats`` is for the backward call."""
    target: object
    entropy: object
    top: object
    top_index: object
    stats: object


def log_probs(logits, targets=None, top: int = 0, scale: float = 1.0) -> LogProbs:
    """Log softmax of ``scale * logits`` at the given classes (-1: none, 0), its entropy and its ``top`` largest entries."""
    torch = _gpu()
    dtype = _rows_of(logits, "logits")
    n, classes = logits.shape
    kind = 0
    if targets is not None:
        kind = _index_code(targets, "targets", logits)
        if targets.shape != (n,):
            raise ValueError(f"targets: shape {tuple(targets.shape)}, expected ({n},)")
    if not 0 <= top <= classes:             # (here, too: it is passed on in 32 bits)
        _check(ERR["SHAPE"], "libra_log_probs")
    nb = libra_log_probs_workspace(n, classes, top)
    device = logits.device
    target = torch.empty(n, dtype=torch.float32, device=device) if targets is not None else None
    entropy = torch.empty(n, dtype=torch.float32, device=device)
    stats = torch.empty(n, 2, dtype=torch.float32, device=device)
    best = torch.empty(n, top, dtype=torch.float32, device=device)
    index = torch.empty(n, top, dtype=torch.int64, device=device)
    ws = torch.empty(nb, dtype=torch.uint8, device=device) if nb else None
    _launch(lib().libra_log_probs, "libra_log_probs", logits, logits.data_ptr(), n, classes, _ld(logits), dtype,
            targets.data_ptr() if targets is not None else 0, kind, top, scale, target.data_ptr() if targets is not None else 0,
            entropy.data_ptr(), best.data_ptr(), index.data_ptr(), stats.data_ptr(), ws.data_ptr() if nb else 0, nb)
    return LogProbs(target, entropy, best, index, stats)


def log_probs_backward(logits, result: LogProbs, targets=None, d_target=None, d_entropy=None, d_top=None, scale: float = 1.0, out=None):
    """Gradient of :func:`log_probs` (its ``result`` for the same logits, targets and scale) with respect to the logits, in their type, from
    the gradients of the target's log probabilities, the entropies and the alternatives' log probabilities (None: zero)."""
    torch = _gpu()
    dtype = _rows_of(logits, "logits")
    n, classes = logits.shape
    top = result.top_index.shape[1]
    kind = 0
    if targets is not None:
        kind = _index_code(targets, "targets", logits)
        if targets.shape != (n,):
            raise ValueError(f"targets: shape {tuple(targets.shape)}, expected ({n},)")
    if d_target is not None and targets is None:
        raise ValueError("d_target: without targets")
    entropy, stats = _fp32_on(result.entropy, "entropy", (n,), logits), _fp32_on(result.stats, "stats", (n, 2), logits)
    if _index_code(result.top_index, "top_index", logits) != INDEX_I64 or result.top_index.shape[0] != n:
        raise ValueError(f"top_index: expected int64 of shape ({n}, top)")
    grads = [0 if t is None else _fp32_on(t, name, want, logits)
             for t, name, want in ((d_target, "d_target", (n,)), (d_entropy, "d_entropy", (n,)), (d_top, "d_top", (n, top)))]
    if out is None:
        out = torch.empty(n, classes, dtype=logits.dtype, device=logits.device)
    else:
        _rows_of(out, "out", classes, like=logits)
        if out.shape[0] != n:
            raise ValueError(f"out: {out.shape[0]} rows, expected {n}")
        _apart(out, logits, "logits")
    _launch(lib().libra_log_probs_backward, "libra_log_probs_backward", logits, logits.data_ptr(), n, classes, _ld(logits), dtype,
            targets.data_ptr() if targets is not None else 0, kind, top, scale, entropy, stats, result.top_index.data_ptr(), *grads,
            out.data_ptr(), _ld(out))
    return out


def _adamw_refuse(k: int, arrays, dtype, n: int, device: int):
    """Says which of the arrays of parameter k is not what it should be: (name, tensor, type, elements) each."""
    for name, t, want, many in arrays:
        if not isinstance(t, _torch.Tensor):
            raise ValueError(f"{name}[{k}]: expected a torch tensor, got {type(t).__name__}")
        if t.dtype is not want or t.numel() != many or not t.is_contiguous() or t.get_device() != device:
            raise ValueError(f"{name}[{k}]: {t.dtype}, {t.numel()} elements, contiguous: {t.is_contiguous()}, {t.device}; expected contiguous "
                             f"{want} of {many} elements on GPU {device}")


def _one_on(x, name: str, dtype, like) -> int:
    """Address of a number that is read on the device when the kernel runs."""
    if x.dtype is not dtype or x.numel() != 1 or x.get_device() != like.get_device():
        raise ValueError(f"{name}: expected one {dtype} on {like.device}")
    return x.data_ptr()


class _AdamwCall(NamedTuple):
    """A step whose tensors have been looked at: what the library takes, and the tensors, which have to live until it has run."""
    table: bytes
    count: int
    opts: AdamwOpts
    params: object
    held: object


def adamw(params, grads, first, second, step, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
          first_scales=None, second_scales=None, masters=None, seed: int = 0, numbers=None):
    """One AdamW step, in place, over lists of contiguous tensors on one GPU.

    ``first``, ``second``: m and v of each parameter in float32; or, with ``first_scales`` and ``second_scales`` (a float32 for every
    ADAMW_BLOCK elements, all given together), m and sqrt(v) in 8 bits, as float8_e4m3fn.  ``masters``: the parameters in float32, of
    which the 16-bit ones are the roundings (a list, None where a tensor has none).  ``step`` counts from 1.  ``step`` and ``lr`` may be
    one-element tensors on the GPU (int64, float32): they are read when the kernel runs, also of a captured step.  ``seed``, ``numbers``
    (of the tensors; their places in the list): of the chances by which 8-bit states are rounded."""
    call = _adamw_checked(params, grads, first, second, step, lr, betas, eps, weight_decay, first_scales, second_scales, masters, seed, numbers)
    if call is not None:
        _adamw_run(call)


def _adamw_run(call: _AdamwCall):
    _launch(lib().libra_adamw, "libra_adamw", call.params[0], call.table, call.count, C.byref(call.opts))
    _torch.autograd.graph.increment_version(call.params)           # a graph that saved one of them must notice


def _adamw_checked(params, grads, first, second, step, lr, betas, eps, weight_decay, first_scales, second_scales, masters, seed, numbers):
    """The call of :func:`adamw` with these arguments; None if there is nothing to do."""
    torch = _gpu()
    count = len(params)
    bits8 = first_scales is not None
    if bits8 != (second_scales is not None):
        raise ValueError("first_scales and second_scales go together")
    for name, x in (("grads", grads), ("first", first), ("second", second), ("first_scales", first_scales), ("second_scales", second_scales),
                    ("masters", masters), ("numbers", numbers)):
        if x is not None and len(x) != count:
            raise ValueError(f"{name}: {len(x)} tensors for {count} parameters")
    if count == 0:
        return None
    state = torch.float8_e4m3fn if bits8 else torch.float32
    device = params[0].get_device()
    if device < 0:
        raise ValueError("params[0]: must be a GPU tensor")
    float32 = torch.float32
    codes = {torch.float16: F16, torch.bfloat16: BF16, float32: F32}
    fields = []                         # a record of AdamwTensor is eight words and two halves of one
    for k, p in enumerate(params):
        g, m, v = grads[k], first[k], second[k]
        ms, vs = (first_scales[k], second_scales[k]) if bits8 else (None, None)
        w = masters[k] if masters is not None else None
        try:
            dtype, n = p.dtype, p.numel()
            blocks = -(-n // ADAMW_BLOCK)
            fine = (dtype in codes and p.is_contiguous() and p.get_device() == device
                    and g.dtype is dtype and g.numel() == n and g.is_contiguous() and g.get_device() == device
                    and m.dtype is state and m.numel() == n and m.is_contiguous() and m.get_device() == device
                    and v.dtype is state and v.numel() == n and v.is_contiguous() and v.get_device() == device
                    and (w is None or w.dtype is float32 and w.numel() == n and w.is_contiguous() and w.get_device() == device)
                    and (not bits8 or ms.dtype is float32 and ms.numel() == blocks and ms.is_contiguous() and ms.get_device() == device
                         and vs.dtype is float32 and vs.numel() == blocks and vs.is_contiguous() and vs.get_device() == device))
        except AttributeError:
            fine = False
        if not fine:
            _code(p, f"params[{k}]")
            n = p.numel()
            more = [("first_scales", ms, float32, -(-n // ADAMW_BLOCK)), ("second_scales", vs, float32, -(-n // ADAMW_BLOCK))] if bits8 else []
            _adamw_refuse(k, [("params", p, p.dtype, n), ("grads", g, p.dtype, n), ("first", m, state, n), ("second", v, state, n), *more,
                              *([("masters", w, float32, n)] if w is not None else [])], p.dtype, n, device)
        number = k if numbers is None else numbers[k] & 0xffffffff
        fields += (p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr(), ms.data_ptr() if bits8 else 0, vs.data_ptr() if bits8 else 0,
                   w.data_ptr() if w is not None else 0, n, codes[dtype] | number << 32)
    if len(set(fields[::9])) < count:
        seen = set()
        for k, p in enumerate(params):
            if p.numel() and p.data_ptr() in seen:
                raise ValueError(f"params[{k}]: the same tensor twice")
            seen.add(p.data_ptr())
    table = struct.pack(f"{len(fields)}Q", *fields)
    opts = AdamwOpts(state_bits=8 if bits8 else 32, beta1=betas[0], beta2=betas[1], eps=eps, weight_decay=weight_decay, seed=seed & 0xffffffff)
    if isinstance(step, torch.Tensor):
        opts.step_dev = _one_on(step, "step", torch.int64, params[0])
    else:
        opts.step = step
    if isinstance(lr, torch.Tensor):
        opts.lr_dev = _one_on(lr, "lr", torch.float32, params[0])
    else:
        opts.lr = lr
    return _AdamwCall(table, count, opts, params, (grads, first, second, first_scales, second_scales, masters, step, lr))
