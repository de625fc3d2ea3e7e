"""Python binding of libgp.so: the same calls as include/gp.h, argument
marshalling only.  Every step of the path runs inside the library's HIP
kernels / host C++; there is no Python or CPU fallback, and a missing library is
an error (build it with `python -m paper_2207_12000_amd.build`).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
from typing import Optional

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


def _on_stream(tensor, stream):
    """Context: the tensor's device and the stream a call is enqueued on (torch's current one unless given) are current while what the
    call needs is allocated, so that torch gives its memory to no other stream before the call is done with it."""
    import torch
    if not tensor.is_cuda:
        raise ValueError("tensors must be on the GPU")
    current = torch.cuda.current_stream(tensor.device).cuda_stream
    handle = current if stream is None else int(stream)
    if handle == current and tensor.device.index == torch.cuda.current_device():
        return contextlib.nullcontext(handle)
    return _other_stream(handle, tensor.device)


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
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("tensors must be on one device")


def _row_stride(t, what):
    """The distance of a matrix's rows, in elements (that of a single row, or of none, is whatever its width asks for)."""
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


def _written(*tensors):
    """Tells torch that a call writes these in place, so that a backward pass that kept what they held is an error."""
    from torch.autograd.graph import increment_version
    increment_version(tensors)


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
