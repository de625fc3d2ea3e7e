"""Python binding of libgp.so: the same calls as include/gp.h, argument
marshalling only.  Every step of the path runs inside the library's HIP
kernels / host C++; there is no Python or CPU fallback, and a missing library is
an error (build it with `python -m paper_2207_12000_amd.build`).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math
import os
from typing import Any, NamedTuple, Optional

import numpy as np

GP_OK = 0
GP_ERR_INVALID_ARG, GP_ERR_INDEX_RANGE, GP_ERR_OVERFLOW = 1, 2, 3
GP_ERR_OOM_HOST, GP_ERR_OOM_DEVICE, GP_ERR_DEVICE, GP_ERR_UNSUPPORTED = 4, 5, 6, 7
GP_AGG_SYM, GP_AGG_MEAN, GP_AGG_SUM = 0, 1, 2
GP_F32, GP_BF16 = 0, 1
GP_SYMMETRISE, GP_ADD_SELF_LOOPS, GP_PLAN_ON_DEVICE = 1, 2, 4

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgp.so")

# every symbol include/gp.h declares: (restype, argtypes)
_c = ctypes
_SIGNATURES = {
    "gp_plan_blocks": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_uint32,
                                  _c.POINTER(_c.c_void_p)]),
    "gp_plan_destroy": (None, [_c.c_void_p]),
    "gp_plan_num_nodes": (_c.c_int64, [_c.c_void_p]),
    "gp_plan_nnz": (_c.c_int64, [_c.c_void_p]),
    "gp_plan_num_blocks": (_c.c_int32, [_c.c_void_p]),
    "gp_plan_block_offsets": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_block_row_lo": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_block_row_hi": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_rowptr": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_col": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_degree": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_dinv_sqrt": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_dinv": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_num_segments": (_c.c_int64, [_c.c_void_p]),
    "gp_plan_segments": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_segment_offsets": (_c.c_void_p, [_c.c_void_p]),
    "gp_plan_num_partial_rows": (_c.c_int64, [_c.c_void_p]),
    "gp_plan_segment_edges": (_c.c_int64, [_c.c_void_p]),
    "gp_plan_row_clusters": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.POINTER(_c.c_int32), _c.POINTER(_c.c_double),
                                        _c.POINTER(_c.c_double)]),
    "gp_plan_work_lists": (_c.c_int, [_c.c_void_p, _c.c_int32, _c.c_int, _c.c_int32, _c.POINTER(_c.c_int32),
                                      _c.POINTER(_c.c_int32), _c.c_void_p, _c.c_void_p, _c.c_int64]),
    "gp_plan_lds_schedule": (_c.c_int, [_c.c_void_p, _c.c_int32, _c.c_int32, _c.c_void_p]),
    "gp_propagate": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int32, _c.c_int, _c.c_int, _c.c_int32,
                                _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_plan_streamed_shape": (_c.c_int, [_c.c_void_p, _c.POINTER(_c.c_int64), _c.POINTER(_c.c_int64)]),
    "gp_propagate_noalloc": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int32, _c.c_int, _c.c_int, _c.c_int32,
                                        _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_noalloc_partial_row_bytes": (_c.c_int64, []),
    "gp_propagate_combine": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int32, _c.c_int, _c.c_int, _c.c_int32,
                                        _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_lc_forward": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_int32, _c.c_void_p, _c.c_int64,
                                 _c.c_void_p, _c.c_int32, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_lc_forward_branches": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_int32, _c.c_void_p,
                                          _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int, _c.c_int32, _c.c_void_p,
                                          _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_lc_softmax": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int32, _c.c_int64, _c.c_void_p]),
    "gp_embedding": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_void_p, _c.c_int, _c.c_int64,
                                _c.c_float, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p]),
    "gp_embedding_grad_workspace": (_c.c_int64, [_c.c_int64, _c.c_int64, _c.c_int32]),
    "gp_embedding_grad": (_c.c_int, [_c.c_void_p, _c.c_int, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_int32, _c.c_float,
                                     _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_int32, _c.c_void_p, _c.c_int64,
                                     _c.c_void_p]),
    "gp_orthogonalize_workspace": (_c.c_int64, [_c.c_int64, _c.c_int64, _c.c_int64]),
    "gp_orthogonalize": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int32,
                                    _c.c_void_p, _c.c_float, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_int64,
                                    _c.c_void_p]),
    "gp_muon_step": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64,
                                _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_float,
                                _c.c_float, _c.c_float, _c.c_int32, _c.c_int32, _c.c_void_p, _c.c_float, _c.c_void_p, _c.c_int64,
                                _c.c_void_p]),
    "gp_layer_norm": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_void_p, _c.c_void_p, _c.c_int, _c.c_float,
                                 _c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_void_p]),
    "gp_layer_norm_grad_workspace": (_c.c_int64, [_c.c_int64, _c.c_int32]),
    "gp_layer_norm_grad": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_void_p,
                                      _c.c_void_p, _c.c_int, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int32, _c.c_void_p,
                                      _c.c_int64, _c.c_void_p]),
    "gp_log_probs_workspace": (_c.c_int64, [_c.c_int64, _c.c_int32, _c.c_int32]),
    "gp_log_probs": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_void_p, _c.c_int, _c.c_float, _c.c_void_p,
                                _c.c_void_p, _c.c_int32, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_log_probs_grad": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_void_p, _c.c_int, _c.c_float, _c.c_void_p,
                                     _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_distill_workspace": (_c.c_int64, [_c.c_int64, _c.c_int32]),
    "gp_distill": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p,
                              _c.c_int64, _c.c_int, _c.c_int32, _c.c_float, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p,
                              _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gp_distill_grad": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int, _c.c_int64, _c.c_int32, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p,
                                   _c.c_int64, _c.c_int, _c.c_int32, _c.c_float, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p,
                                   _c.c_int64, _c.c_void_p]),
    "gp_solve_normalisation_blocks": (_c.c_int, [_c.c_double] * 7 + [_c.POINTER(_c.c_int64)]),
    "gp_solve_aggregation_blocks": (_c.c_int, [_c.c_double] * 5 + [_c.c_int64, _c.POINTER(_c.c_int64),
                                                                  _c.POINTER(_c.c_int64)]),
    "gp_set_hbm_budget_bytes": (_c.c_int, [_c.c_int64]),
    "gp_set_option": (_c.c_int, [_c.c_char_p, _c.c_int64]),
    "gp_get_option": (_c.c_int64, [_c.c_char_p]),
    "gp_profile_enable": (_c.c_int, [_c.c_int32]),
    "gp_profile_read": (_c.c_int, [_c.c_char_p, _c.POINTER(_c.c_int64), _c.POINTER(_c.c_double)]),
    "gp_status_string": (_c.c_char_p, [_c.c_int]),
    "gp_last_error": (_c.c_char_p, []),
}
EXPORTED_SYMBOLS = tuple(_SIGNATURES)

_lib = None


class GpError(RuntimeError):
    def __init__(self, status: int, where: str):
        l = lib()
        self.status = status
        self.status_name = l.gp_status_string(status).decode()
        super().__init__(f"{where}: {self.status_name}: {l.gp_last_error().decode()}")


def lib():
    """Loads libgp.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2207_12000_amd.build`")
        # PyTorch brings a HIP runtime of its own and loads it for the whole process.  Loaded after this
        # library's, the process holds two runtimes that each open the GPU, and calls through the second
        # fail ("no ROCm-capable device is detected"); loaded before, this library's calls resolve to the
        # runtime that is already there.  So PyTorch goes first wherever it is installed.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


def _check(status: int, where: str):
    if status != GP_OK:
        raise GpError(status, where)


def _view(ptr, ctype, count, dtype):
    if not ptr or count == 0:
        return np.empty(0, dtype=dtype)
    return np.ctypeslib.as_array(ctypes.cast(ptr, ctypes.POINTER(ctype)), shape=(count,))


class Plan:
    """Owns a gp_plan*.  The array properties are views of library-owned host
    memory, valid until close()."""

    def __init__(self, handle: int):
        self._h = handle

    @property
    def handle(self) -> int:
        if not self._h:
            raise ValueError("plan is closed")
        return self._h

    def close(self):
        if self._h:
            lib().gp_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    @property
    def n(self) -> int:
        return lib().gp_plan_num_nodes(self.handle)

    @property
    def nnz(self) -> int:
        return lib().gp_plan_nnz(self.handle)

    @property
    def num_blocks(self) -> int:
        return lib().gp_plan_num_blocks(self.handle)

    @property
    def block_off(self):
        return _view(lib().gp_plan_block_offsets(self.handle), ctypes.c_int64, self.num_blocks + 1, np.int64)

    @property
    def block_row_lo(self):
        return _view(lib().gp_plan_block_row_lo(self.handle), ctypes.c_int32, self.num_blocks, np.int32)

    @property
    def block_row_hi(self):
        return _view(lib().gp_plan_block_row_hi(self.handle), ctypes.c_int32, self.num_blocks, np.int32)

    @property
    def rowptr(self):
        return _view(lib().gp_plan_rowptr(self.handle), ctypes.c_int64, self.n + 1, np.int64)

    @property
    def col(self):
        return _view(lib().gp_plan_col(self.handle), ctypes.c_int32, self.nnz, np.int32)

    @property
    def deg(self):
        return _view(lib().gp_plan_degree(self.handle), ctypes.c_int32, self.n, np.int32)

    @property
    def dinv_sqrt(self):
        return _view(lib().gp_plan_dinv_sqrt(self.handle), ctypes.c_float, self.n, np.float32)

    @property
    def dinv(self):
        return _view(lib().gp_plan_dinv(self.handle), ctypes.c_float, self.n, np.float32)


    SEGMENT_DTYPE = np.dtype([("start_lo", "<u4"), ("start_hi", "u1"), ("slice", "u1"), ("len", "<u2"),
                              ("row", "<i4"), ("slot", "<i4")])

    @property
    def segments(self):
        """Structured view of the schedule's 16-byte segment records."""
        cnt = lib().gp_plan_num_segments(self.handle)
        raw = _view(lib().gp_plan_segments(self.handle), ctypes.c_uint8, cnt * 16, np.uint8)
        return raw.view(self.SEGMENT_DTYPE)

    @property
    def segment_off(self):
        return _view(lib().gp_plan_segment_offsets(self.handle), ctypes.c_int64, self.num_blocks + 1, np.int64)

    @property
    def num_partial_rows(self) -> int:
        return lib().gp_plan_num_partial_rows(self.handle)

    @property
    def segment_edges(self) -> int:
        return lib().gp_plan_segment_edges(self.handle)

    def streamed_shape(self):
        """(edge blocks b, column blocks c) of the last streamed gp_propagate on this plan."""
        b, c = ctypes.c_int64(), ctypes.c_int64()
        _check(lib().gp_plan_streamed_shape(self.handle, ctypes.byref(b), ctypes.byref(c)), "gp_plan_streamed_shape")
        return b.value, c.value

    def row_clusters(self):
        """(label[n], num_clusters, inside_fraction, typical_rows) of the cache schedule."""
        label = np.empty(self.n, dtype=np.int32)
        num, inside, typical = ctypes.c_int32(), ctypes.c_double(), ctypes.c_double()
        _check(lib().gp_plan_row_clusters(self.handle, label.ctypes.data, ctypes.byref(num), ctypes.byref(inside),
                                          ctypes.byref(typical)), "gp_plan_row_clusters")
        return label, num.value, inside.value, typical.value

    def work_lists(self, d: int, dtype: int, vec: int):
        """(num_slices, slice_elems, xcd_off[9], records) of the explicit work lists for rows of
        d elements, or num_slices = 0 when the plan keeps the implicit lists."""
        S, elems = ctypes.c_int32(), ctypes.c_int32()
        off = np.zeros(9, dtype=np.int64)
        _check(lib().gp_plan_work_lists(self.handle, d, dtype, vec, ctypes.byref(S), ctypes.byref(elems), off.ctypes.data,
                                        None, 0), "gp_plan_work_lists")
        recs = np.zeros(int(off[8]), dtype=self.SEGMENT_DTYPE)
        if S.value:
            _check(lib().gp_plan_work_lists(self.handle, d, dtype, vec, ctypes.byref(S), ctypes.byref(elems),
                                            off.ctypes.data, recs.ctypes.data, recs.size), "gp_plan_work_lists")
        return S.value, elems.value, off, recs

    def lds_schedule(self, order: int = 0, d: int = 128):
        """The LDS pass's schedule (see gp_plan_lds_schedule in gp.h), or None where it does not
        apply: dict with hot_mode, conflict_free, group_set, group_id_off, group_steps (per
        group), rec_pos (64 per group), ids (uint16 places on the set's list), list_of_set,
        member_off, members, rest (segment records in position order), col (reordered)."""
        v = LdsView()
        _check(lib().gp_plan_lds_schedule(self.handle, d, order, ctypes.byref(v)), "gp_plan_lds_schedule")
        if v.num_groups == 0:
            return None
        G = v.num_groups
        out = {"group_set": np.zeros(G, np.int32), "group_id_off": np.zeros(G, np.int64), "group_steps": np.zeros(G, np.int32),
               "rec_pos": np.zeros(G * 64, np.int32), "ids": np.zeros(v.num_ids, np.uint16),
               "list_of_set": np.zeros(v.num_sets, np.int32), "member_off": np.zeros(v.num_lists + 1, np.int64),
               "members": np.zeros(v.num_members, np.int32), "rest": np.zeros(v.num_positions, self.SEGMENT_DTYPE),
               "col": np.zeros(self.nnz, np.int32)}
        v.group_capacity, v.id_capacity, v.member_capacity = G, v.num_ids, v.num_members
        v.set_capacity = max(v.num_sets, v.num_lists + 1)
        v.position_capacity = max(v.num_positions, self.nnz)
        for k, a in out.items():
            setattr(v, k, a.ctypes.data)
        _check(lib().gp_plan_lds_schedule(self.handle, d, order, ctypes.byref(v)), "gp_plan_lds_schedule")
        out["conflict_free"] = bool(v.conflict_free)
        out["hot_mode"] = int(v.hot_mode)
        return out


class LdsView(ctypes.Structure):
    """gp_lds_view of gp.h."""
    _fields_ = [("num_groups", ctypes.c_int64), ("num_ids", ctypes.c_int64), ("num_members", ctypes.c_int64),
                ("num_positions", ctypes.c_int64),
                ("num_sets", ctypes.c_int32), ("num_lists", ctypes.c_int32), ("conflict_free", ctypes.c_int32),
                ("hot_mode", ctypes.c_int32),
                ("group_capacity", ctypes.c_int64), ("id_capacity", ctypes.c_int64), ("set_capacity", ctypes.c_int64),
                ("member_capacity", ctypes.c_int64), ("position_capacity", ctypes.c_int64),
                ("group_set", ctypes.c_void_p), ("group_id_off", ctypes.c_void_p), ("group_steps", ctypes.c_void_p),
                ("rec_pos", ctypes.c_void_p), ("ids", ctypes.c_void_p),
                ("list_of_set", ctypes.c_void_p), ("member_off", ctypes.c_void_p), ("members", ctypes.c_void_p),
                ("rest", ctypes.c_void_p), ("col", ctypes.c_void_p)]


def gp_plan_blocks(src, dst, n: int, block_budget_edges: int, flags: int) -> Plan:
    """src/dst: int32 host arrays (numpy) of equal length."""
    src = np.ascontiguousarray(src, dtype=np.int32)
    dst = np.ascontiguousarray(dst, dtype=np.int32)
    if src.shape != dst.shape or src.ndim != 1:
        raise ValueError("src and dst must be 1-D and equally long")
    out = ctypes.c_void_p()
    st = lib().gp_plan_blocks(src.ctypes.data if src.size else None, dst.ctypes.data if dst.size else None,
                              src.size, n, block_budget_edges, flags, ctypes.byref(out))
    _check(st, "gp_plan_blocks")
    return Plan(out.value)


def gp_propagate(plan: Plan, X_ptr: int, ldx: int, d: int, dtype: int, agg: int, K: int, out_ptr: int, ldo: int,
                 stream: Optional[int] = None):
    """Raw-pointer form: X_ptr / out_ptr are device (or pinned host) addresses."""
    st = lib().gp_propagate(plan.handle, X_ptr, ldx, d, dtype, agg, K, out_ptr, ldo, stream or None)
    _check(st, "gp_propagate")


def gp_propagate_noalloc(plan: Plan, X_ptr: int, ldx: int, d: int, dtype: int, agg: int, K: int, out_ptr: int, ldo: int,
                         stream: Optional[int] = None):
    """gp_propagate without any allocation (device operands, plan already on the device)."""
    st = lib().gp_propagate_noalloc(plan.handle, X_ptr, ldx, d, dtype, agg, K, out_ptr, ldo, stream or None)
    _check(st, "gp_propagate_noalloc")


def gp_noalloc_partial_row_bytes() -> int:
    return lib().gp_noalloc_partial_row_bytes()


def gp_propagate_combine(plan: Plan, X_ptr: int, ldx: int, d: int, dtype: int, agg: int, K: int, coeff, out_ptr: int,
                         ldo: int, stream: Optional[int] = None):
    """coeff: K+1 host floats.  X_ptr / out_ptr: device addresses."""
    c = np.ascontiguousarray(coeff, dtype=np.float32)
    if c.shape != (K + 1,):
        raise ValueError("coeff must hold K+1 values")
    st = lib().gp_propagate_combine(plan.handle, X_ptr, ldx, d, dtype, agg, K, c.ctypes.data, out_ptr, ldo, stream or None)
    _check(st, "gp_propagate_combine")


def propagate_tensors(plan: Plan, X, agg: int, K: int, out=None, stream=None):
    """Convenience for torch tensors (memory and streams only): X is an (n, d)
    float32 or bfloat16 tensor on the GPU (or pinned host memory); returns the
    (K+1, n, d) stack.  Enqueued on torch's current stream unless given."""
    import torch
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be 2-D with unit column stride")
    n, d = X.shape
    if n != plan.n:
        raise ValueError("X has the wrong number of rows")
    dtype = {torch.float32: GP_F32, torch.bfloat16: GP_BF16}[X.dtype]
    if out is None:
        out = torch.empty((K + 1, n, d), dtype=X.dtype, device=X.device,
                          pin_memory=(X.device.type == "cpu"))
    if out.shape != (K + 1, n, d) or out.dtype != X.dtype or not out.is_contiguous():
        raise ValueError("out must be a contiguous (K+1, n, d) tensor of X's dtype")
    if stream is None and X.is_cuda:
        stream = torch.cuda.current_stream(X.device).cuda_stream
    gp_propagate(plan, X.data_ptr(), X.stride(0), d, dtype, agg, K, out.data_ptr(), d, stream)
    return out


def gp_lc_forward(stack_ptr: int, ld: int, dtype: int, n: int, d: int, K: int, batch_ptr: Optional[int], B: int, gamma,
                  weight_ptrs, widths, out_ptr: int, ldo: int, stream: Optional[int] = None):
    """Raw-pointer form.  gamma: K+1 host floats; weight_ptrs: T device addresses;
    widths: T output widths; batch_ptr: device address of B int32 row numbers or None."""
    g = np.ascontiguousarray(gamma, dtype=np.float32)
    if g.shape != (K + 1,):
        raise ValueError("gamma must hold K+1 values")
    T = len(weight_ptrs)
    if len(widths) != T:
        raise ValueError("one width per weight matrix")
    W = (ctypes.c_void_p * max(T, 1))(*[int(p) for p in weight_ptrs])
    wd = np.ascontiguousarray(widths, dtype=np.int32)
    st = lib().gp_lc_forward(stack_ptr, ld, dtype, n, d, K, batch_ptr or None, B, g.ctypes.data, T,
                             ctypes.cast(W, ctypes.c_void_p), wd.ctypes.data, out_ptr, ldo, stream or None)
    _check(st, "gp_lc_forward")


GP_COMB_SUM, GP_COMB_CONCAT, GP_COMB_MAX = 0, 1, 2


def gp_lc_softmax(H_ptr: int, B: int, C: int, ld: int, stream: Optional[int] = None):
    """Row softmax in place on a device matrix of B x C floats (rows ld floats apart)."""
    _check(lib().gp_lc_softmax(H_ptr or None, B, C, ld, stream or None), "gp_lc_softmax")


def gp_lc_forward_branches(stack_ptr: int, ld: int, dtype: int, n: int, d: int, K: int, batch_ptr: Optional[int], B: int,
                           gamma, depth, comb: int, weight_ptrs, widths, out_ptr: int, ldo: int,
                           stream: Optional[int] = None):
    """Raw-pointer form.  depth: K+1 host ints (layers branch k applies, 0 = hop left out);
    comb: GP_COMB_SUM / GP_COMB_CONCAT / GP_COMB_MAX; the rest as gp_lc_forward."""
    g = np.ascontiguousarray(gamma, dtype=np.float32)
    dp = np.ascontiguousarray(depth, dtype=np.int32)
    if g.shape != (K + 1,) or dp.shape != (K + 1,):
        raise ValueError("gamma and depth must hold K+1 values")
    T = len(weight_ptrs)
    if len(widths) != T:
        raise ValueError("one width per weight matrix")
    W = (ctypes.c_void_p * max(T, 1))(*[int(p) for p in weight_ptrs])
    wd = np.ascontiguousarray(widths, dtype=np.int32)
    st = lib().gp_lc_forward_branches(stack_ptr, ld, dtype, n, d, K, batch_ptr or None, B, g.ctypes.data, dp.ctypes.data, comb,
                                      T, ctypes.cast(W, ctypes.c_void_p), wd.ctypes.data, out_ptr, ldo, stream or None)
    _check(st, "gp_lc_forward_branches")


def lc_forward_tensors(stack, batch, gamma, weights, out=None, stream=None, depth=None, comb=GP_COMB_SUM):
    """Convenience for torch tensors (memory and streams only): stack is the
    contiguous (K+1, n, d) float32 / bfloat16 GPU tensor gp_propagate filled, batch an
    int32 GPU tensor of row numbers (or None for all rows), weights a list of
    contiguous float32 GPU matrices.  Returns the (B, width) float32 result.  With
    `depth` (K+1 ints) the branch form gp_lc_forward_branches is called."""
    import torch
    if stack.dim() != 3 or not stack.is_contiguous():
        raise ValueError("stack must be a contiguous (K+1, n, d) tensor")
    K1, n, d = stack.shape
    dtype = {torch.float32: GP_F32, torch.bfloat16: GP_BF16}[stack.dtype]
    if batch is not None and (batch.dtype != torch.int32 or batch.dim() != 1 or not batch.is_contiguous()):
        raise ValueError("batch must be a contiguous int32 vector")
    B = n if batch is None else batch.numel()
    inner = d
    for W in weights:
        if W.dtype != torch.float32 or W.dim() != 2 or not W.is_contiguous() or W.shape[0] != inner:
            raise ValueError("weights must be contiguous float32 matrices whose shapes chain from d")
        inner = W.shape[1]
    if depth is not None:
        ends = [weights[dk - 1].shape[1] for dk in depth if dk > 0]
        if not ends:
            raise ValueError("every hop is left out")
        inner = sum(ends) if comb == GP_COMB_CONCAT else ends[0]
    if out is None:
        out = torch.empty((B, inner), dtype=torch.float32, device=stack.device)
    if out.shape != (B, inner) or out.dtype != torch.float32 or out.stride(1) != 1:
        raise ValueError("out must be a (B, width) float32 tensor with unit column stride")
    if stream is None:
        stream = torch.cuda.current_stream(stack.device).cuda_stream
    bp = None if batch is None else batch.data_ptr()
    wp, ww = [W.data_ptr() for W in weights], [W.shape[1] for W in weights]
    if depth is None:
        gp_lc_forward(stack.data_ptr(), d, dtype, n, d, K1 - 1, bp, B, gamma, wp, ww, out.data_ptr(), out.stride(0), stream)
    else:
        gp_lc_forward_branches(stack.data_ptr(), d, dtype, n, d, K1 - 1, bp, B, gamma, depth, comb, wp, ww, out.data_ptr(),
                               out.stride(0), stream)
    return out


GP_I32, GP_I64 = 0, 1


def gp_embedding(table_ptr: int, ldt: int, dtype: int, V: int, d: int, tokens_ptr: int, index: int, N: int, scale: float,
                 out_ptr: int, ldo: int, out_dtype: int, stream: Optional[int] = None):
    """Raw-pointer form: out[i, :] = scale * table[token[i], :]; all addresses are device addresses."""
    st = lib().gp_embedding(table_ptr or None, ldt, dtype, V, d, tokens_ptr or None, index, N, scale, out_ptr or None, ldo,
                            out_dtype, stream or None)
    _check(st, "gp_embedding")


def gp_embedding_grad_workspace(N: int, V: int, d: int) -> int:
    return lib().gp_embedding_grad_workspace(N, V, d)


def gp_embedding_grad(tokens_ptr: int, index: int, N: int, grad_ptr: int, ldg: int, dtype: int, d: int, scale: float, V: int,
                      table_grad_ptr: int, ldt: int, out_dtype: int, accumulate: bool, workspace_ptr: int, workspace_bytes: int,
                      stream: Optional[int] = None):
    """Raw-pointer form of the gradient of gp_embedding; all addresses are device addresses."""
    st = lib().gp_embedding_grad(tokens_ptr or None, index, N, grad_ptr or None, ldg, dtype, d, scale, V, table_grad_ptr or None,
                                 ldt, out_dtype, int(accumulate), workspace_ptr or None, workspace_bytes, stream or None)
    _check(st, "gp_embedding_grad")


def gp_orthogonalize_workspace(rows: int, cols: int, count: int = 1) -> int:
    return lib().gp_orthogonalize_workspace(rows, cols, count)


def _coefficients(coeff, steps: int):
    """(steps, 3) host floats from one triple for all steps, one for each, or None (the library's own)."""
    if coeff is None:
        return None
    c = np.ascontiguousarray(coeff, dtype=np.float32)
    if c.shape == (3,):
        c = np.ascontiguousarray(np.broadcast_to(c, (max(steps, 0), 3)))
    if c.shape != (steps, 3):
        raise ValueError("coeff must hold three values, or three for every step")
    return c


def gp_orthogonalize(G_ptr: int, ldg: int, stride_g: int, dtype: int, rows: int, cols: int, count: int, steps: int, coeff, eps: float,
                     out_ptr: int, ldo: int, stride_o: int, workspace_ptr: int, workspace_bytes: int, stream: Optional[int] = None):
    """Raw-pointer form.  coeff: three host floats, three for every step, or None."""
    c = _coefficients(coeff, steps)
    st = lib().gp_orthogonalize(G_ptr or None, ldg, stride_g, dtype, rows, cols, count, steps, None if c is None else c.ctypes.data,
                                eps, out_ptr or None, ldo, stride_o, workspace_ptr or None, workspace_bytes, stream or None)
    _check(st, "gp_orthogonalize")


def gp_muon_step(W_ptr: int, W_out_ptr: int, ldw: int, stride_w: int, M_ptr: int, M_out_ptr: int, ldm: int, stride_m: int, G_ptr: int,
                 ldg: int, stride_g: int, dtype: int, rows: int, cols: int, count: int, lr: float, momentum: float,
                 weight_decay: float, nesterov: bool, steps: int, coeff, eps: float, workspace_ptr: int, workspace_bytes: int,
                 stream: Optional[int] = None):
    """Raw-pointer form.  coeff: three host floats, three for every step, or None."""
    c = _coefficients(coeff, steps)
    st = lib().gp_muon_step(W_ptr or None, W_out_ptr or None, ldw, stride_w, M_ptr or None, M_out_ptr or None, ldm, stride_m,
                            G_ptr or None, ldg, stride_g, dtype, rows, cols, count, lr, momentum, weight_decay, int(nesterov), steps,
                            None if c is None else c.ctypes.data, eps, workspace_ptr or None, workspace_bytes, stream or None)
    _check(st, "gp_muon_step")


@contextlib.contextmanager
def _other_stream(handle, device):
    import torch
    with torch.cuda.stream(torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)):
        yield handle


@functools.lru_cache(maxsize=None)
def _current():
    """(the handle of a device's current stream by its number, the current device, whether torch records a trace, torch's forward mode): 1.7 us of a call's 11
    are spent on torch's stream object, where its handle cannot be had without one."""
    import torch
    bare = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return (bare or (lambda index: torch.cuda.current_stream(index).cuda_stream), torch.cuda.current_device,
            getattr(torch._C, "_is_tracing", torch.jit.is_tracing), torch.autograd.forward_ad)


_TRACED = "torch.jit.trace would record a result's memory and not the call that fills it"


def _on_stream(tensor, stream):
    """Context: the tensor's device and the stream a call is enqueued on (torch's current one unless given) are current while what the
    call needs is allocated, so that torch gives its memory to no other stream before the call is done with it."""
    current_handle, current_device, tracing, _ = _current()
    if tracing():
        raise ValueError(_TRACED)
    if not tensor.is_cuda:
        raise ValueError("tensors must be on the GPU")
    index = tensor.get_device()
    current = current_handle(index)
    handle = current if stream is None else int(stream)
    if handle == current and index == current_device():
        return contextlib.nullcontext(handle)
    return _other_stream(handle, tensor.device)


def _no_tangent(*tensors):
    """Derivatives in forward mode are not followed: a tensor that carries one is refused, as the result would be without."""
    forward = _current()[3]
    if getattr(forward, "_current_level", 0) >= 0 and any(t is not None and forward.unpack_dual(t).tangent is not None for t in tensors):
        raise ValueError("forward-mode derivatives are not followed: give the primal tensors")


@functools.lru_cache(maxsize=None)
def _types():
    import torch
    return {torch.float32: GP_F32, torch.bfloat16: GP_BF16}, {torch.int32: GP_I32, torch.int64: GP_I64}


def _float_type(t):
    kind = _types()[0].get(t.dtype)
    if kind is None:
        raise ValueError("values must be float32 or bfloat16")
    return kind


def _index_type(tokens):
    kind = _types()[1].get(tokens.dtype)
    if kind is None or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous int32 or int64 tensor")
    return kind


def _one_device(first, *others):
    device = first.device
    for t in others:
        if t is not None and t.device != device:
            raise ValueError("tensors must be on one device")


def _row_stride(t, what):
    """The distance of a matrix's rows, in elements (that of a single row, or of none, is whatever its width asks for)."""
    if t.is_contiguous():
        return max(t.shape[-1], 1)
    if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel() > 0:
        raise ValueError(f"{what} must have unit column stride")
    return max(t.shape[-1], 1) if t.shape[-2] <= 1 else t.stride(-2)


def _workspace(workspace, need, device):
    import torch
    if workspace is None:
        return torch.empty(max(need, 0), dtype=torch.uint8, device=device)
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor")
    return workspace


@functools.lru_cache(maxsize=None)
def _increment_version():
    from torch.autograd.graph import increment_version
    return increment_version


def _written(*tensors):
    """Tells torch that a call writes these in place, so that a backward pass that kept what they held is an error."""
    _increment_version()(tensors)


def _new_like(t, dtype=None):
    """A contiguous tensor of t's shape and device, of its type unless another is given."""
    import torch
    if dtype in (None, t.dtype) and t.is_contiguous():
        return torch.empty_like(t)
    return torch.empty(t.shape, dtype=dtype or t.dtype, device=t.device)


@functools.lru_cache(maxsize=None)
def _differentiable_lookup():
    import torch

    class Lookup(torch.autograd.Function):
        @staticmethod
        def forward(ctx, table, tokens, scale, out_dtype, stream):
            ctx.save_for_backward(tokens)
            ctx.scale, ctx.shape, ctx.dtype = scale, table.shape, table.dtype
            return embedding_tensors(table, tokens, scale, out_dtype=out_dtype, stream=stream)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad):
            tokens, = ctx.saved_tensors
            V, d = ctx.shape
            grad = grad.reshape(tokens.numel(), d)
            if (d > 1 and grad.stride(1) != 1) or 0 < grad.stride(0) < d:  # (a sum's gradient is one number, expanded)
                grad = grad.contiguous()
            return embedding_grad_tensors(tokens, grad, V, ctx.scale, out_dtype=ctx.dtype), None, None, None, None

    return Lookup


def embedding_tensors(table, tokens, scale=1.0, out=None, out_dtype=None, stream=None):
    """Convenience for torch tensors: table is a (V, d) float32 / bfloat16 GPU tensor, tokens an int32 / int64 GPU tensor of
    any shape.  Returns scale * table[tokens], of shape tokens.shape + (d,), in out_dtype (the table's unless given); a
    token outside the table gives zeros.  out: a (tokens.numel(), d) tensor with unit column stride, filled and returned.
    Where the table requires a gradient, the result does too: backward() takes it by embedding_grad_tensors, on the stream that was
    current here.  What is filled into out is a plain copy that automatic differentiation does not follow."""
    import torch
    _no_tangent(table)
    if out is None and table.requires_grad and torch.is_grad_enabled():
        return _differentiable_lookup().apply(table, tokens, scale, out_dtype, stream)
    if table.dim() != 2:
        raise ValueError("table must be a (V, d) tensor")
    V, d = table.shape
    dtype, index, ldt = _float_type(table), _index_type(tokens), _row_stride(table, "table")
    N = tokens.numel()
    if out is not None and (out.dim() != 2 or out.shape != (N, d) or out_dtype not in (None, out.dtype)):
        raise ValueError("out must be a (tokens, d) tensor of out_dtype")
    _one_device(table, tokens, out)
    with _on_stream(table, stream) as handle:
        result = out
        if out is None:
            result = torch.empty(tuple(tokens.shape) + (d,), dtype=out_dtype or table.dtype, device=table.device)
            out = result.view(N, d)
        else:
            _written(out)
        gp_embedding(table.data_ptr(), ldt, dtype, V, d, tokens.data_ptr(), index, N, scale, out.data_ptr(), _row_stride(out, "out"),
                     _float_type(out), handle)
    return result


def embedding_grad_tensors(tokens, grad, V, scale=1.0, out=None, out_dtype=None, accumulate=False, workspace=None, stream=None):
    """Convenience for torch tensors: the gradient of embedding_tensors with respect to its table of V rows, from grad, the
    gradient of what it returned ((N, d), or tokens.shape + (d,) contiguous).  Returns a (V, d) tensor of out_dtype (grad's
    unless given; automatic differentiation does not follow it), or adds to out (accumulate=True).  workspace: a uint8 GPU tensor of gp_embedding_grad_workspace(N, V, d)
    bytes or more, kept by the caller; without one the call takes its memory from torch."""
    import torch
    N, index, dtype = tokens.numel(), _index_type(tokens), _float_type(grad)
    if grad.dim() != 2:
        if grad.dim() == 0 or tuple(grad.shape[:-1]) != tuple(tokens.shape) or not grad.is_contiguous():
            raise ValueError("grad of other than two dimensions must be contiguous, of shape tokens.shape + (d,)")
        grad = grad.view(N, grad.shape[-1])
    if grad.shape[0] != N:
        raise ValueError("grad must hold one row per token")
    d = grad.shape[1]
    if accumulate and out is None:
        raise ValueError("accumulate needs a tensor to add to")
    if out is not None and (out.dim() != 2 or out.shape != (V, d) or out_dtype not in (None, out.dtype)):
        raise ValueError("out must be a (V, d) tensor of out_dtype")
    _one_device(tokens, grad, out, workspace)
    with _on_stream(grad, stream) as handle:
        if out is None:
            out = torch.empty((V, d), dtype=out_dtype or grad.dtype, device=grad.device)
        else:
            _written(out)
        ws = _workspace(workspace, gp_embedding_grad_workspace(N, V, d), grad.device)
        gp_embedding_grad(tokens.data_ptr(), index, N, grad.data_ptr(), _row_stride(grad, "grad"), dtype, d, scale, V, out.data_ptr(),
                          _row_stride(out, "out"), _float_type(out), accumulate, ws.data_ptr(), ws.numel(), handle)
    return out


def _matrices(t, shape, dtype, what):
    """(rows, cols, count, row distance, matrix distance) of a (rows, cols) or (count, rows, cols) tensor."""
    if t.dim() not in (2, 3) or (shape is not None and t.shape != shape) or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{what} must be a (rows, cols) or (count, rows, cols) tensor, all of one shape, of the right type")
    count = t.shape[0] if t.dim() == 3 else 1
    return t.shape[-2], t.shape[-1], count, _row_stride(t, what), t.stride(0) if t.dim() == 3 and count > 1 else 0


def orthogonalize_tensors(G, steps=5, coeff=None, eps=1e-7, out=None, workspace=None, stream=None):
    """Convenience for torch tensors: Newton-Schulz steps on G, a (rows, cols) or (count, rows, cols) float32 / bfloat16 GPU
    tensor.  coeff: (a, b, c), or three for every step, or None (3.4445, -4.7750, 2.0315).  Returns out (made if not given;
    G itself will do); automatic differentiation does not follow it.  workspace: a uint8 GPU tensor of gp_orthogonalize_workspace(rows, cols, count) bytes or more."""
    import torch
    rows, cols, count, ldg, sg = _matrices(G, None, None, "G")
    dtype = _float_type(G)
    if out is not None:
        _matrices(out, G.shape, G.dtype, "out")
    _one_device(G, out, workspace)
    with _on_stream(G, stream) as handle:
        if out is None:
            out = torch.empty(G.shape, dtype=G.dtype, device=G.device)
        else:
            _written(out)
        _, _, _, ldo, so = _matrices(out, G.shape, G.dtype, "out")
        ws = _workspace(workspace, gp_orthogonalize_workspace(rows, cols, count), G.device)
        gp_orthogonalize(G.data_ptr(), ldg, sg, dtype, rows, cols, count, steps, coeff, eps, out.data_ptr(), ldo, so, ws.data_ptr(),
                         ws.numel(), handle)
    return out


def muon_step_tensors(W, M, G, lr, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, coeff=None, eps=1e-7, W_out=None,
                      M_out=None, workspace=None, stream=None):
    """Convenience for torch tensors: one step of weight matrices W (float32) with momentum M (float32) and gradient G (float32 /
    bfloat16), all (rows, cols) or (count, rows, cols).  W and M are stepped in place unless W_out, M_out are given (of the
    same strides; torch's version counters see it).  Returns (W_out, M_out).  coeff, workspace: as orthogonalize_tensors."""
    import torch
    rows, cols, count, ldg, sg = _matrices(G, None, None, "G")
    dtype = _float_type(G)
    W_out, M_out = W if W_out is None else W_out, M if M_out is None else M_out
    _, _, _, ldw, sw = _matrices(W, G.shape, torch.float32, "W")
    _, _, _, ldm, sm = _matrices(M, G.shape, torch.float32, "M")
    if _matrices(W_out, G.shape, torch.float32, "W_out")[3:] != (ldw, sw) or _matrices(M_out, G.shape, torch.float32, "M_out")[3:] != (ldm, sm):
        raise ValueError("W_out and M_out must have the strides of W and M")
    _one_device(G, W, M, W_out, M_out, workspace)
    with _on_stream(G, stream) as handle:
        _written(W_out, M_out)
        ws = _workspace(workspace, gp_orthogonalize_workspace(rows, cols, count), G.device)
        gp_muon_step(W.data_ptr(), W_out.data_ptr(), ldw, sw, M.data_ptr(), M_out.data_ptr(), ldm, sm, G.data_ptr(), ldg, sg, dtype, rows,
                     cols, count, lr, momentum, weight_decay, nesterov, steps, coeff, eps, ws.data_ptr(), ws.numel(), handle)
    return W_out, M_out


def gp_layer_norm(x_ptr: int, ldx: int, dtype: int, N: int, d: int, weight_ptr: Optional[int], bias_ptr: Optional[int], weight_dtype: int,
                  eps: float, y_ptr: int, ldy: int, out_dtype: int, stats_ptr: Optional[int] = None, stream: Optional[int] = None):
    """Raw-pointer form: y = (x - mean) / sqrt(variance + eps) * weight + bias row by row; all addresses are device addresses."""
    st = lib().gp_layer_norm(x_ptr or None, ldx, dtype, N, d, weight_ptr or None, bias_ptr or None, weight_dtype, eps, y_ptr or None, ldy,
                             out_dtype, stats_ptr or None, stream or None)
    _check(st, "gp_layer_norm")


@functools.lru_cache(maxsize=256)  # (of the sizes alone)
def gp_layer_norm_grad_workspace(N: int, d: int) -> int:
    return lib().gp_layer_norm_grad_workspace(N, d)


def gp_layer_norm_grad(grad_ptr: int, ldg: int, grad_dtype: int, x_ptr: int, ldx: int, dtype: int, N: int, d: int, stats_ptr: int,
                       weight_ptr: Optional[int], weight_dtype: int, x_grad_ptr: Optional[int], ldxg: int, weight_grad_ptr: Optional[int],
                       bias_grad_ptr: Optional[int], accumulate: bool, workspace_ptr: int, workspace_bytes: int, stream: Optional[int] = None):
    """Raw-pointer form of the gradients of gp_layer_norm; all addresses are device addresses."""
    st = lib().gp_layer_norm_grad(grad_ptr or None, ldg, grad_dtype, x_ptr or None, ldx, dtype, N, d, stats_ptr or None, weight_ptr or None,
                                  weight_dtype, x_grad_ptr or None, ldxg, weight_grad_ptr or None, bias_grad_ptr or None, int(accumulate),
                                  workspace_ptr or None, workspace_bytes, stream or None)
    _check(st, "gp_layer_norm_grad")


@functools.lru_cache(maxsize=256)  # (of the sizes alone)
def gp_log_probs_workspace(N: int, C: int, k: int = 0) -> int:
    return lib().gp_log_probs_workspace(N, C, k)


def gp_log_probs(logits_ptr: int, ld: int, dtype: int, N: int, C: int, tokens_ptr: Optional[int], index: int, scale: float,
                 logp_ptr: Optional[int], entropy_ptr: Optional[int], k: int, top_index_ptr: Optional[int], top_logp_ptr: Optional[int],
                 stats_ptr: Optional[int], workspace_ptr: Optional[int], workspace_bytes: int, stream: Optional[int] = None):
    """Raw-pointer form; all addresses are device addresses."""
    st = lib().gp_log_probs(logits_ptr or None, ld, dtype, N, C, tokens_ptr or None, index, scale, logp_ptr or None, entropy_ptr or None, k,
                            top_index_ptr or None, top_logp_ptr or None, stats_ptr or None, workspace_ptr or None, workspace_bytes,
                            stream or None)
    _check(st, "gp_log_probs")


def gp_log_probs_grad(logits_ptr: int, ld: int, dtype: int, N: int, C: int, tokens_ptr: Optional[int], index: int, scale: float,
                      stats_ptr: int, entropy_ptr: Optional[int], grad_logp_ptr: Optional[int], stride_logp: int,
                      grad_entropy_ptr: Optional[int], stride_entropy: int, grad_ptr: int, ldg: int, stream: Optional[int] = None):
    """Raw-pointer form of the gradient of gp_log_probs; all addresses are device addresses."""
    st = lib().gp_log_probs_grad(logits_ptr or None, ld, dtype, N, C, tokens_ptr or None, index, scale, stats_ptr or None, entropy_ptr or None,
                                 grad_logp_ptr or None, stride_logp, grad_entropy_ptr or None, stride_entropy, grad_ptr or None, ldg,
                                 stream or None)
    _check(st, "gp_log_probs_grad")


@functools.lru_cache(maxsize=256)  # (of the sizes alone)
def gp_distill_workspace(N: int, C: int) -> int:
    return lib().gp_distill_workspace(N, C)


def gp_distill(logits_ptr: int, ld: int, dtype: int, N: int, C: int, teacher_index_ptr: int, ldi: int, index: int, teacher_logits_ptr: int,
               ldt: int, teacher_dtype: int, K: int, temperature: float, loss_ptr: Optional[int], stats_ptr: Optional[int],
               grad_loss_ptr: Optional[int], stride_loss: int, grad_ptr: Optional[int], ldg: int, workspace_ptr: Optional[int],
               workspace_bytes: int, stream: Optional[int] = None):
    """Raw-pointer form; all addresses are device addresses."""
    st = lib().gp_distill(logits_ptr or None, ld, dtype, N, C, teacher_index_ptr or None, ldi, index, teacher_logits_ptr or None, ldt,
                          teacher_dtype, K, temperature, loss_ptr or None, stats_ptr or None, grad_loss_ptr or None, stride_loss,
                          grad_ptr or None, ldg, workspace_ptr or None, workspace_bytes, stream or None)
    _check(st, "gp_distill")


def gp_distill_grad(logits_ptr: int, ld: int, dtype: int, N: int, C: int, teacher_index_ptr: int, ldi: int, index: int,
                    teacher_logits_ptr: int, ldt: int, teacher_dtype: int, K: int, temperature: float, stats_ptr: int, grad_loss_ptr: int,
                    stride_loss: int, grad_ptr: int, ldg: int, stream: Optional[int] = None):
    """Raw-pointer form of the gradient of gp_distill from the stats that it left; all addresses are device addresses."""
    st = lib().gp_distill_grad(logits_ptr or None, ld, dtype, N, C, teacher_index_ptr or None, ldi, index, teacher_logits_ptr or None, ldt,
                               teacher_dtype, K, temperature, stats_ptr or None, grad_loss_ptr or None, stride_loss, grad_ptr or None, ldg,
                               stream or None)
    _check(st, "gp_distill_grad")


def _followed(t, stream):
    """Whether automatic differentiation is to follow a call on t.  Its backward pass runs on the stream that is current at the call, and may meet
    leaves that a graph outside a capture has as well, which ends the process: so neither another stream nor a capture goes with it."""
    if t is None or not t.requires_grad:
        return False
    import torch
    if not torch.is_grad_enabled():
        return False
    if _current()[2]():
        raise ValueError(_TRACED)
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    if stream is not None:
        raise ValueError("a call that automatic differentiation follows runs on the current stream: set that one")
    with contextlib.nullcontext() if t.get_device() == torch.cuda.current_device() else torch.cuda.device(t.device):
        capturing = torch.cuda.is_current_stream_capturing()
    if capturing:
        raise ValueError("a call that automatic differentiation follows is not captured: capture it under torch.no_grad(), and the gradient's own call")
    return True


def _not_captured():
    """A backward pass in a capture may meet leaves that a graph outside it has as well, which ends the process: the gradient's own calls can be captured."""
    import torch
    if torch.cuda.is_current_stream_capturing():
        raise ValueError("a backward pass is not captured: capture the gradient's own call")


def _as_rows(t, what):
    """A (rows, width) view of a tensor whose last dimension is a row: any distance of rows in two dimensions, contiguous in others."""
    if t.dim() == 2:
        return t
    if t.dim() == 0 or not t.is_contiguous() or t.shape[-1] == 0:
        raise ValueError(f"{what} of other than two dimensions must be contiguous, its last dimension a row")
    return t.view(-1, t.shape[-1])


def _rows_for(t, shape, dtype, what):
    """(view, distance of rows) of a tensor that rows are written to: of `shape`, or two-dimensional with as many rows."""
    if (t.shape != shape and tuple(t.shape) != (math.prod(shape[:-1]), shape[-1])) or t.dtype != dtype:
        raise ValueError(f"{what} must be of the rows' shape and of the right type")
    t = _as_rows(t, what)
    return t, _row_stride(t, what)


def _memory(t):
    """(address, bytes from row to row, bytes of a row, rows) of what a tensor takes; a contiguous one is a single row."""
    size = t.element_size()
    if t.dim() == 2 and t.stride(0) > 0 and not t.is_contiguous():
        return t.data_ptr(), t.stride(0) * size, ((t.shape[1] - 1) * t.stride(1) + 1) * size, t.shape[0]
    return t.data_ptr(), 0, (sum((n - 1) * step for n, step in zip(t.shape, t.stride())) + 1) * size, 1


def _overlap(a, b):
    """Whether two tensors share memory.  Rows of one distance may lie between each other's, as columns of one matrix do; of two distances they may not."""
    if a.numel() == 0 or b.numel() == 0:
        return False
    (p, step, width, rows), (q, other_step, other_width, other_rows) = _memory(a), _memory(b)
    if p >= q + (other_rows - 1) * other_step + other_width or q >= p + (rows - 1) * step + width:
        return False
    if rows > 1 and other_rows > 1 and step != other_step:
        return True
    if other_rows == 1:
        (p, step, width, rows), (q, other_step, other_width, other_rows) = (q, other_step, other_width, other_rows), (p, step, width, rows)
    if other_rows == 1:
        return True
    past = (p - q) % other_step  # of the other's rows that the first begins in or behind
    return past < other_width or past + width > other_step


def _end(t):
    address, step, width, rows = _memory(t)
    return address + (rows - 1) * step + width


def _clear(*tensors):
    """Whether no two tensors share memory, as far as their ends tell (None: left out)."""
    last = 0
    for at, end in sorted([(t.data_ptr(), t.data_ptr() + t.nbytes if t.is_contiguous() else _end(t)) for t in tensors if t is not None]):
        if at < last:
            return False
        last = end
    return True


def _apart(out, what, *inputs):
    """Refuses a tensor to write that shares memory with what is read: another workgroup may read there after it was written."""
    start = out.data_ptr()
    end = start + out.nbytes if out.is_contiguous() else _end(out)
    for t in inputs:
        if t is None:
            continue
        at = t.data_ptr()
        if at < end and not (at < start and t.is_contiguous() and at + t.nbytes <= start) and _overlap(out, t):
            raise ValueError(f"{what} must not overlap what the call reads or writes besides")


def _itself(out, t):
    """Whether a call that writes out over t writes every element over itself (both matrices)."""
    return out.data_ptr() == t.data_ptr() and out.dtype == t.dtype and out.shape == t.shape and (out.stride() == t.stride() or out.is_contiguous() and t.is_contiguous())


def _vector(t, n, what):
    if t is not None and (t.dim() != 1 or t.shape[0] != n or not t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous vector, one value per column")


def _row_stats(stats, N):
    import torch
    if stats is not None and (stats.dtype != torch.float32 or tuple(stats.shape) != (N, 2) or not stats.is_contiguous()):
        raise ValueError("stats must be a contiguous (rows, 2) float32 tensor")


def _per_row(t, N, what):
    """(tensor, distance of its elements) of a float32 value per row, or of one that stands for all rows."""
    import torch
    if t is None:
        return None, 0
    if t.dtype != torch.float32:
        raise ValueError(f"{what} must be float32")
    if t.numel() == 1 or (t.numel() == N and not any(t.stride()) and N > 0):
        return t, 0
    if t.numel() != N or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous, one value per row, or one for all")
    return t, 1


def _ptr(t):
    return None if t is None else t.data_ptr()


@functools.lru_cache(maxsize=None)
def _differentiable_norm():
    import torch

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, eps, out_dtype):
            stats = torch.empty((x.numel() // max(x.shape[-1], 1), 2), dtype=torch.float32, device=x.device)
            y = layer_norm_tensors(x, weight, bias, eps, out_dtype=out_dtype, stats=stats)
            ctx.save_for_backward(x, weight, stats)
            ctx.weight_dtype = None if weight is None and bias is None else (bias if weight is None else weight).dtype
            return y

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad):
            _not_captured()
            x, weight, stats = ctx.saved_tensors
            want = ctx.needs_input_grad
            rows = grad.reshape(-1, x.shape[-1])
            if (rows.shape[1] > 1 and rows.stride(1) != 1) or 0 < rows.stride(0) < rows.shape[1]:  # (a sum's gradient is one number, expanded)
                rows = rows.contiguous()
            x_grad, weight_grad, bias_grad = layer_norm_grad_tensors(rows, _as_rows(x, "x"), stats, weight, x_grad=None if want[0] else False,
                                                                     weight_grad=None if want[1] else False, bias_grad=None if want[2] else False,
                                                                     weight_dtype=ctx.weight_dtype)
            return None if x_grad is None else x_grad.view(x.shape), weight_grad, bias_grad, None, None

    return Norm


def layer_norm_tensors(x, weight=None, bias=None, eps=1e-5, out=None, out_dtype=None, stats=None, stream=None):
    """Convenience for torch tensors: x is a float32 / bfloat16 GPU tensor whose last dimension is normalised (any distance of rows in two dimensions,
    contiguous in others), weight and bias vectors of float32 or bfloat16 (both of one type) or None.  Returns the normalised rows, of x's shape,
    in out_dtype (x's unless given); out: a tensor of that shape, filled and returned (x itself will do, else it must not overlap the inputs).  stats: a (rows, 2) float32 tensor that
    receives what layer_norm_grad_tensors needs.  Where x, weight or bias require a gradient, the result does too (not with out, stats or a stream of
    its own, nor in a capture)."""
    _no_tangent(x, weight, bias)
    if out is None and stats is None and (_followed(x, stream) or _followed(weight, stream) or _followed(bias, stream)):
        return _differentiable_norm().apply(x, weight, bias, eps, out_dtype)
    dtype, rows = _float_type(x), _as_rows(x, "x")
    N, d = rows.shape
    ldx = _row_stride(rows, "x")
    _vector(weight, d, "weight")
    _vector(bias, d, "bias")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must be of one type")
    kind = weight if weight is not None else bias
    weight_dtype = GP_F32 if kind is None else _float_type(kind)
    _row_stats(stats, N)
    if out is not None:
        to, ldy = _rows_for(out, x.shape, out_dtype or out.dtype, "out")
    _one_device(x, weight, bias, out, stats)
    if out is not None:
        _apart(to, "out", weight, bias, stats, None if _itself(to, rows) else rows)
    with _on_stream(x, stream) as handle:
        if out is None:
            out = _new_like(x, out_dtype)
            to, ldy = out, d
        else:
            _written(out)
        if stats is not None:
            _written(stats)
        gp_layer_norm(x.data_ptr(), ldx, dtype, N, d, _ptr(weight), _ptr(bias), weight_dtype, eps, to.data_ptr(), ldy, _float_type(out), _ptr(stats),
                      handle)
    return out


def layer_norm_grad_tensors(grad, x, stats, weight=None, x_grad=None, weight_grad=None, bias_grad=None, accumulate=False, weight_dtype=None,
                            workspace=None, stream=None):
    """Convenience for torch tensors: the gradients of layer_norm_tensors from grad, the gradient of what it returned, and the stats it left.  Returns
    (x_grad, weight_grad, bias_grad): each is made where None is given, filled where a tensor is, left out (None) where False is.  What is filled must not
    overlap the inputs or each other, but for x_grad, which may be x or grad itself, and weight's and bias's, which may be written over weight.  accumulate: weight_grad
    and bias_grad are added to (both given, or False).  weight_dtype: of the gradients that are made (weight's; float32 without one).  workspace: a uint8
    GPU tensor of gp_layer_norm_grad_workspace(rows, d) bytes or more, kept by the caller; without one the call takes its memory from torch.  Automatic
    differentiation does not follow it."""
    import torch
    dtype, grad_dtype = _float_type(x), _float_type(grad)
    rows, up = _as_rows(x, "x"), _as_rows(grad, "grad")
    if rows.shape != up.shape:
        raise ValueError("grad must be of x's shape")
    N, d = rows.shape
    ldx = _row_stride(rows, "x")
    ldg = _row_stride(up, "grad")
    _row_stats(stats, N)
    if stats is None:
        raise ValueError("stats are needed")
    _vector(weight, d, "weight")
    given = [t for t in (weight, weight_grad, bias_grad) if t is not None and t is not False]
    weight_dtype = weight_dtype or (given[0].dtype if given else torch.float32)
    if any(t.dtype != weight_dtype for t in given):
        raise ValueError("weight and the gradients of weight and bias must be of one type")
    if accumulate and (weight_grad is None or bias_grad is None):
        raise ValueError("accumulate needs tensors to add to")
    for t, what in ((weight_grad, "weight_grad"), (bias_grad, "bias_grad")):
        if t is not False:
            _vector(t, d, what)
    if x_grad is not None and x_grad is not False:
        to, ldxg = _rows_for(x_grad, x.shape, x.dtype, "x_grad")
    outs = [None if t is False else t for t in (x_grad, weight_grad, bias_grad)]
    _one_device(x, grad, stats, weight, workspace, *outs)
    given = [t for t in outs if t is not None]
    other = [t for t in (rows, up) if outs[0] is None or not _itself(to, t)]
    over_weight = False
    if given and not _clear(*given, *other, stats, weight):
        if outs[0] is not None:
            _apart(to, "x_grad", *other, stats, weight)
        sums = [t for t in outs[1:] if t is not None]
        for i, t in enumerate(sums):
            _apart(t, "weight_grad or bias_grad", rows, up, stats, outs[0], *sums[:i])
        over_weight = weight is not None and any(_overlap(t, weight) for t in sums)
    with _on_stream(x, stream) as handle:
        if given:
            _written(*given)
        if x_grad is None:
            x_grad = _new_like(x)
            to, ldxg = x_grad, d
        elif x_grad is False:
            x_grad, to, ldxg = None, None, d
        if weight_grad is None:
            weight_grad = torch.empty(d, dtype=weight_dtype, device=x.device) if weight is None else _new_like(weight)
        if bias_grad is None:
            bias_grad = torch.empty(d, dtype=weight_dtype, device=x.device) if weight is None else _new_like(weight)
        weight_grad, bias_grad = (None if t is False else t for t in (weight_grad, bias_grad))
        need = gp_layer_norm_grad_workspace(N, d)
        ws = _workspace(workspace, need, x.device) if need > 0 else None
        kind = _types()[0].get(weight_dtype, -1)
        if over_weight:
            weight = weight.detach().clone()  # (few rows: workgroups that read it run beside those that write its gradient)
        gp_layer_norm_grad(up.data_ptr(), ldg, grad_dtype, rows.data_ptr(), ldx, dtype, N, d, stats.data_ptr(), _ptr(weight), kind, _ptr(to), ldxg,
                           _ptr(weight_grad), _ptr(bias_grad), accumulate, _ptr(ws), 0 if ws is None else ws.numel(), handle)
    return x_grad, weight_grad, bias_grad


class LogProbs(NamedTuple):
    """What log_probs_tensors returns; None in the place of what was not asked for."""
    logp: Any
    entropy: Any
    top_index: Any
    top_logp: Any


def _rows_of_logits(logits, tokens):
    rows = _as_rows(logits, "logits")
    if tokens is not None and tokens.shape != logits.shape[:-1]:
        raise ValueError("tokens must hold one class per row")
    return rows, _row_stride(rows, "logits")


@functools.lru_cache(maxsize=None)
def _differentiable_log_probs():
    import torch

    class Answers(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, tokens, scale, top, entropy, workspace):
            stats = torch.empty((logits.numel() // max(logits.shape[-1], 1), 2), dtype=torch.float32, device=logits.device)
            a = log_probs_tensors(logits, tokens, scale, top, entropy, stats=stats, workspace=workspace)
            ctx.save_for_backward(logits, tokens, stats, a.entropy)
            ctx.scale = scale
            if top:
                ctx.mark_non_differentiable(a.top_index, a.top_logp)
            ctx.set_materialize_grads(False)
            return tuple(a)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad_logp, grad_entropy, _index, _top):
            _not_captured()
            logits, tokens, stats, entropy = ctx.saved_tensors
            grads = [None if g is None else g if g.is_contiguous() or not any(g.stride()) else g.contiguous() for g in (grad_logp, grad_entropy)]
            return log_probs_grad_tensors(logits, tokens, stats, ctx.scale, entropy, *grads), None, None, None, None, None

    return Answers


def log_probs_tensors(logits, tokens=None, scale=1.0, top=0, entropy=True, stats=None, workspace=None, stream=None):
    """Convenience for torch tensors: logits is a float32 / bfloat16 GPU tensor whose last dimension holds the classes (any distance of rows in two
    dimensions, contiguous in others), tokens an int32 / int64 GPU tensor of one class per row.  Returns LogProbs(logp, entropy, top_index, top_logp)
    of scale * logits: the tokens' log probabilities (0 where a token is outside the classes), the rows' entropies, and the `top` (up to 64) best
    classes (int32) with their log probabilities; ties go to the lower class.  stats: a (rows, 2) float32 tensor that receives what
    log_probs_grad_tensors needs.  workspace: a uint8 GPU tensor of gp_log_probs_workspace(rows, classes, top) bytes or more, kept by the caller.  Where
    logits require a gradient, logp and entropy do too (not with stats or a stream of its own, nor in a capture)."""
    import torch
    _no_tangent(logits)
    if stats is None and _followed(logits, stream):
        return LogProbs(*_differentiable_log_probs().apply(logits, tokens, scale, top, entropy, workspace))
    dtype, index = _float_type(logits), GP_I32 if tokens is None else _index_type(tokens)
    rows, ld = _rows_of_logits(logits, tokens)
    N, C = rows.shape
    _row_stats(stats, N)
    if top < 0:
        raise ValueError("top must be 0 or more")
    _one_device(logits, tokens, stats, workspace)
    with _on_stream(logits, stream) as handle:
        if stats is not None:
            _written(stats)
        shape, device = logits.shape[:-1], logits.device
        logp = None if tokens is None else torch.empty(shape, dtype=torch.float32, device=device)
        spread = None if not entropy else torch.empty(shape, dtype=torch.float32, device=device) if logp is None else torch.empty_like(logp)
        best = torch.empty((*shape, top), dtype=torch.int32, device=device) if top else None
        best_logp = torch.empty((*shape, top), dtype=torch.float32, device=device) if top else None
        need = gp_log_probs_workspace(N, C, top)
        ws = _workspace(workspace, need, logits.device) if need > 0 else None
        gp_log_probs(rows.data_ptr(), ld, dtype, N, C, _ptr(tokens), index, scale, _ptr(logp), _ptr(spread), top, _ptr(best), _ptr(best_logp),
                     _ptr(stats), _ptr(ws), 0 if ws is None else ws.numel(), handle)
    return LogProbs(logp, spread, best, best_logp)


def log_probs_grad_tensors(logits, tokens, stats, scale=1.0, entropy=None, grad_logp=None, grad_entropy=None, out=None, stream=None):
    """Convenience for torch tensors: the gradient of log_probs_tensors with respect to its logits, from the stats (and, for grad_entropy, the entropy) it left.
    grad_logp, grad_entropy: float32, one value per row or one for all, or None.  Returns out, of logits' shape and type (made if not given; it must not
    overlap the inputs); automatic differentiation does not follow it."""
    dtype, index = _float_type(logits), GP_I32 if tokens is None else _index_type(tokens)
    rows, ld = _rows_of_logits(logits, tokens)
    N, C = rows.shape
    if stats is None:
        raise ValueError("stats are needed")
    _row_stats(stats, N)
    grad_logp, s1 = _per_row(grad_logp, N, "grad_logp")
    grad_entropy, s2 = _per_row(grad_entropy, N, "grad_entropy")
    if grad_entropy is not None and (entropy is None or _per_row(entropy, N, "entropy")[1] != (1 if N != 1 else 0)):
        raise ValueError("the entropies are needed, one per row")
    if grad_logp is not None and tokens is None:
        raise ValueError("tokens are needed")
    if out is not None:
        to, ldg = _rows_for(out, logits.shape, logits.dtype, "out")
    _one_device(logits, tokens, stats, entropy, grad_logp, grad_entropy, out)
    if out is not None:
        _apart(to, "out", rows, tokens, stats, entropy, grad_logp, grad_entropy)
    with _on_stream(logits, stream) as handle:
        if out is None:
            out = _new_like(logits)
            to, ldg = out, C
        else:
            _written(out)
        gp_log_probs_grad(rows.data_ptr(), ld, dtype, N, C, _ptr(tokens), index, scale, stats.data_ptr(), _ptr(entropy), _ptr(grad_logp), s1,
                          _ptr(grad_entropy), s2, to.data_ptr(), ldg, handle)
    return out


def _teacher(logits, teacher_index, teacher_logits):
    """(address, distance of rows, type) of a teacher's classes and of their logits, and the entries of a row."""
    if teacher_index.shape[:-1] != logits.shape[:-1] or teacher_index.shape != teacher_logits.shape:
        raise ValueError("teacher_index and teacher_logits must be of one shape, with a row for every row of logits")
    index = _types()[1].get(teacher_index.dtype)
    if index is None:
        raise ValueError("teacher_index must be int32 or int64")
    at, values = _as_rows(teacher_index, "teacher_index"), _as_rows(teacher_logits, "teacher_logits")
    return (at.data_ptr(), _row_stride(at, "teacher_index"), index, values.data_ptr(), _row_stride(values, "teacher_logits"),
            _float_type(teacher_logits), at.shape[1])


@functools.lru_cache(maxsize=None)
def _differentiable_distill():
    import torch

    class Distill(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, teacher_index, teacher_logits, temperature, workspace):
            stats = torch.empty((logits.numel() // max(logits.shape[-1], 1), 2), dtype=torch.float32, device=logits.device)
            loss = distill_tensors(logits, teacher_index, teacher_logits, temperature, stats=stats, workspace=workspace)
            ctx.save_for_backward(logits, teacher_index, teacher_logits, stats)
            ctx.temperature = temperature
            return loss

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad):
            _not_captured()
            logits, teacher_index, teacher_logits, stats = ctx.saved_tensors
            grad = grad if grad.is_contiguous() or not any(grad.stride()) else grad.contiguous()
            return distill_grad_tensors(logits, teacher_index, teacher_logits, stats, grad, ctx.temperature), None, None, None, None

    return Distill


def distill_tensors(logits, teacher_index, teacher_logits, temperature=1.0, grad_loss=None, out=None, stats=None, workspace=None, stream=None):
    """Convenience for torch tensors: the loss of every row of logits (as log_probs_tensors takes them) against a teacher's best classes and their logits, each
    one row of up to 64 per row of logits (int32 / int64, -1 for none, and float32 / bfloat16: log_probs_tensors' top_index and top_logp will do).  Returns the
    float32 losses, of logits.shape[:-1]; with grad_loss (float32, one value per row or one for all) the gradient of the logits is made in the same
    pass and (loss, gradient) returned, the gradient in out where that is given (not over the inputs).  stats: a (rows, 2) float32 tensor that receives what
    distill_grad_tensors needs.  workspace: a uint8 GPU tensor of gp_distill_workspace(rows, classes) bytes or more, kept by the caller.  Where logits
    require a gradient, the loss does too (not with grad_loss, stats or a stream of its own, nor in a capture); the teacher gets none."""
    import torch
    _no_tangent(logits, teacher_logits)
    if stats is None and grad_loss is None and _followed(logits, stream):
        return _differentiable_distill().apply(logits, teacher_index, teacher_logits, temperature, workspace)
    dtype = _float_type(logits)
    rows, ld = _rows_of_logits(logits, None)
    N, C = rows.shape
    at, ldi, index, values, ldt, teacher_dtype, K = _teacher(logits, teacher_index, teacher_logits)
    _row_stats(stats, N)
    if out is not None and grad_loss is None:
        raise ValueError("out takes a gradient, which needs grad_loss")
    grad_loss, stride = _per_row(grad_loss, N, "grad_loss")
    to, ldg = (None, C) if out is None else _rows_for(out, logits.shape, logits.dtype, "out")
    _one_device(logits, teacher_index, teacher_logits, grad_loss, out, stats, workspace)
    if out is not None:
        _apart(to, "out", rows, teacher_index, teacher_logits, grad_loss, stats)
    with _on_stream(logits, stream) as handle:
        loss = torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)
        if out is not None:
            _written(out)
        elif grad_loss is not None:
            to = out = _new_like(logits)
        if stats is not None:
            _written(stats)
        need = gp_distill_workspace(N, C)
        ws = _workspace(workspace, need, logits.device) if need > 0 else None
        gp_distill(rows.data_ptr(), ld, dtype, N, C, at, ldi, index, values, ldt, teacher_dtype, K, temperature, loss.data_ptr(), _ptr(stats),
                   _ptr(grad_loss), stride, _ptr(to), ldg, _ptr(ws), 0 if ws is None else ws.numel(), handle)
    return loss if grad_loss is None else (loss, out)


def distill_grad_tensors(logits, teacher_index, teacher_logits, stats, grad_loss, temperature=1.0, out=None, stream=None):
    """Convenience for torch tensors: the gradient of distill_tensors with respect to its logits, from the stats it left and grad_loss, the gradient of the
    losses (float32, one value per row or one for all).  Returns out, of logits' shape and type (made if not given; it must not overlap the inputs);
    automatic differentiation does not follow it."""
    dtype = _float_type(logits)
    rows, ld = _rows_of_logits(logits, None)
    N, C = rows.shape
    at, ldi, index, values, ldt, teacher_dtype, K = _teacher(logits, teacher_index, teacher_logits)
    if stats is None or grad_loss is None:
        raise ValueError("stats and grad_loss are needed")
    _row_stats(stats, N)
    grad_loss, stride = _per_row(grad_loss, N, "grad_loss")
    if out is not None:
        to, ldg = _rows_for(out, logits.shape, logits.dtype, "out")
    _one_device(logits, teacher_index, teacher_logits, stats, grad_loss, out)
    if out is not None:
        _apart(to, "out", rows, teacher_index, teacher_logits, stats, grad_loss)
    with _on_stream(logits, stream) as handle:
        if out is None:
            out = _new_like(logits)
            to, ldg = out, C
        else:
            _written(out)
        gp_distill_grad(rows.data_ptr(), ld, dtype, N, C, at, ldi, index, values, ldt, teacher_dtype, K, temperature, stats.data_ptr(),
                        grad_loss.data_ptr(), stride, to.data_ptr(), ldg, handle)
    return out


def gp_solve_normalisation_blocks(B_A, B_S, B_D, B_GPU, alpha_A=1.0, alpha_S=1.0, alpha_D=1.0) -> int:
    a = ctypes.c_int64()
    _check(lib().gp_solve_normalisation_blocks(B_A, B_S, B_D, B_GPU, alpha_A, alpha_S, alpha_D, ctypes.byref(a)),
           "gp_solve_normalisation_blocks")
    return a.value


def gp_solve_aggregation_blocks(B_S, B_X, B_GPU, beta_S=1.0, beta_X=1.0, max_c=1 << 20):
    b, c = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().gp_solve_aggregation_blocks(B_S, B_X, B_GPU, beta_S, beta_X, max_c, ctypes.byref(b), ctypes.byref(c)),
           "gp_solve_aggregation_blocks")
    return b.value, c.value


def gp_set_hbm_budget_bytes(nbytes: int):
    _check(lib().gp_set_hbm_budget_bytes(nbytes), "gp_set_hbm_budget_bytes")


def gp_set_option(name: str, value: int):
    _check(lib().gp_set_option(name.encode(), value), "gp_set_option")


def gp_get_option(name: str) -> int:
    return lib().gp_get_option(name.encode())


def gp_profile_enable(on: bool):
    _check(lib().gp_profile_enable(1 if on else 0), "gp_profile_enable")


def gp_profile_read(prefix: str = ""):
    n = ctypes.c_int64()
    ms = ctypes.c_double()
    _check(lib().gp_profile_read(prefix.encode(), ctypes.byref(n), ctypes.byref(ms)), "gp_profile_read")
    return n.value, ms.value


def gp_status_string(status: int) -> str:
    return lib().gp_status_string(status).decode()


def gp_last_error() -> str:
    return lib().gp_last_error().decode()
