"""ctypes binding of libdbsp's C ABI (include/dbsp.h): argument marshalling only.

Every step of the hot path runs inside the library; nothing here computes.  The library is
loaded from this package's directory; if it has not been built yet it is built once with
hipcc, and any failure to build or load raises -- there is no CPU fallback.
"""

from __future__ import annotations

import copy
import ctypes as C
import os
import struct

import numpy as np

from . import build as _build

DBSP_OK, DBSP_EINVAL, DBSP_ESHAPE, DBSP_ENOMEM, DBSP_EHIP = 0, -1, -2, -3, -4
MODE_BALANCED, MODE_NAIVE, MODE_ROUNDS, MODE_REWARD = 0, 1, 2, 3
PLAN_HOST_ONLY = 1
PLAN_PAIR_ROWS = 2
PLAN_PAIR_AUTO = 4

ROW_PTR, KV_IDX, ITEMS, ITEM_SLOT, SPLIT_ROWS, PART_PTR, PART_ITEMS, PART_LOAD, BLOCKS_PER_HEAD, ROW_CNT, EMPTY_ROWS, TAIL_ITEMS = range(12)
_INT64_ARRAYS = (PART_LOAD, BLOCKS_PER_HEAD)

EXPORTS = (
    "plan_sparse_attn", "plan_sparse_attn_reuse", "sparse_attn_fwd", "sparse_attn_fwd_static", "imbalance_ratio", "dbsp_plan_get", "dbsp_plan_stats",
    "dbsp_plan_busy", "dbsp_plan_tail_takes", "dbsp_plan_pair_rows", "dbsp_plan_calibrate", "dbsp_plan_destroy", "dbsp_plan_release", "dbsp_last_error",
    "dbsp_partition_heads", "dbsp_partition_blocks", "dbsp_ring_work", "dbsp_fit_cost_model", "dbsp_mfma_probe", "dbsp_plan_run_order",
    "dbsp_cache_attn_fwd", "dbsp_cache_attn_workspace", "dbsp_cache_evict", "dbsp_cache_evict_workspace",
    "dbsp_cache_attn_layout",
    "dbsp_qk_norm_rope_fwd", "dbsp_qk_norm_rope_bwd", "dbsp_qk_norm_rope_bwd_workspace",
    "dbsp_paged_append", "dbsp_paged_attn_fwd", "dbsp_paged_attn_workspace",
)


class DbspError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libdbsp error {code}: {msg}")
        self.code = code


class PlanOpts(C.Structure):
    _fields_ = [("num_partitions", C.c_int32), ("mode", C.c_int32), ("max_item_len", C.c_int32),
                ("item_overhead", C.c_int32), ("flags", C.c_int32), ("locality_groups", C.c_int32),
                ("partition_cost", C.c_void_p), ("max_batch", C.c_int32), ("dynamic_tail", C.c_int32), ("reward", C.c_double),
                ("head_dim", C.c_int32)]


class CacheDesc(C.Structure):
    """dbsp_cache of dbsp.h."""
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("Hk", C.c_int32), ("d", C.c_int32), ("n_prefix", C.c_int32), ("capacity", C.c_int32),
                ("prefix_k", C.c_void_p), ("prefix_v", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
                ("prefix_k_stride", C.c_int64 * 2), ("prefix_v_stride", C.c_int64 * 2), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("lens", C.c_void_p), ("weights", C.c_void_p), ("positions", C.c_void_p)]


class CacheLayout(C.Structure):
    """dbsp_cache_layout of dbsp_diag.h."""
    _fields_ = [(name, C.c_int32) for name in ("many", "pooled", "joined", "join_by_row", "row_tiles", "cut", "parts", "longest_first", "scores_kept", "weight_parts")]


class HeadNormDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("gains_f32", C.c_int32), ("eps", C.c_float), ("q_gain", C.c_void_p), ("k_gain", C.c_void_p),
                ("q_bias", C.c_void_p), ("k_bias", C.c_void_p)]


class RotaryDesc(C.Structure):
    _fields_ = [("axes", C.c_int32), ("halves", C.c_int32), ("pairs", C.c_int32 * 4), ("freqs", C.POINTER(C.c_double))]


# dbsp_heads and dbsp_qk_rows of dbsp.h, packed in one call: a structure's fields cost as much as an argument each.
_HEADS = struct.Struct("@P3q")
_QK_ROWS = struct.Struct("@6i" + "P3q" * 4 + "P2q")
_NO_HEADS = (0, 0, 0, 0)
_NO_POSITIONS = (0, 0, 0)


class PagedCacheDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("Hk", C.c_int32), ("d", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("max_pages", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("pages", C.c_void_p), ("pages_stride", C.c_int64), ("lens", C.c_void_p)]


_lib = None
_torch = None      # torch, once a forward call has needed it


def load_library(path: str | None = None):
    """Load libdbsp.so (building it first if it does not exist).  Raises if that fails."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or _build.LIB_PATH
    if not os.path.exists(path):
        _build.build()
    lib = C.CDLL(path)
    vp, i32, i64p = C.c_void_p, C.c_int32, C.POINTER(C.c_int64)
    lib.plan_sparse_attn.argtypes = [vp, i32, i32, i32, i32, C.POINTER(PlanOpts), C.POINTER(vp)]
    lib.plan_sparse_attn.restype = C.c_int
    lib.plan_sparse_attn_reuse.argtypes = [vp, vp, C.POINTER(PlanOpts), C.c_double, C.POINTER(vp), C.POINTER(C.c_int32), C.POINTER(C.c_double)]
    lib.plan_sparse_attn_reuse.restype = C.c_int
    i32, i64, f64 = C.c_int32, C.c_int64, C.c_double
    lib.dbsp_partition_heads.argtypes = [vp, i32, i32, i32, vp, f64, vp, vp, vp, vp, C.POINTER(f64), C.POINTER(f64), C.POINTER(f64), C.POINTER(i32)]
    lib.dbsp_partition_heads.restype = C.c_int
    lib.dbsp_partition_blocks.argtypes = [vp, i32, i32, i32, i32, f64, i32, i32, vp, vp, vp, vp, vp, vp, vp,
                                          C.POINTER(f64), C.POINTER(f64), C.POINTER(i64), C.POINTER(i64)]
    lib.dbsp_partition_blocks.restype = C.c_int
    lib.dbsp_ring_work.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, C.POINTER(f64)]
    lib.dbsp_ring_work.restype = C.c_int
    lib.dbsp_fit_cost_model.argtypes = [vp, vp, vp, i32, C.POINTER(f64), C.POINTER(f64), C.POINTER(f64), C.POINTER(f64)]
    lib.dbsp_fit_cost_model.restype = C.c_int
    lib.dbsp_mfma_probe.argtypes = [C.POINTER(f64), C.POINTER(f64), vp]
    lib.dbsp_mfma_probe.restype = C.c_int
    lib.dbsp_plan_calibrate.argtypes = [vp, vp, vp]
    lib.dbsp_plan_calibrate.restype = C.c_int
    lib.sparse_attn_fwd.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, C.c_float, vp]
    lib.sparse_attn_fwd.restype = C.c_int
    lib.sparse_attn_fwd_static.argtypes = lib.sparse_attn_fwd.argtypes
    lib.sparse_attn_fwd_static.restype = C.c_int
    lib.imbalance_ratio.argtypes = [vp, i32, i32, C.POINTER(C.c_double)]
    lib.imbalance_ratio.restype = C.c_int
    lib.dbsp_plan_get.argtypes = [vp, i32, C.POINTER(vp), i64p]
    lib.dbsp_plan_get.restype = C.c_int
    lib.dbsp_plan_stats.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double), i64p, i64p,
                                    C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_double)]
    lib.dbsp_plan_stats.restype = C.c_int
    lib.dbsp_plan_busy.argtypes = [vp, vp, vp, vp]
    lib.dbsp_plan_busy.restype = C.c_int
    lib.dbsp_plan_tail_takes.argtypes = [vp, vp, vp]
    lib.dbsp_plan_tail_takes.restype = C.c_int
    lib.dbsp_plan_pair_rows.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.dbsp_plan_pair_rows.restype = C.c_int
    lib.dbsp_plan_run_order.argtypes = [vp, vp, vp, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.dbsp_plan_run_order.restype = C.c_int
    cache, f32 = C.POINTER(CacheDesc), C.c_float
    lib.dbsp_cache_attn_fwd.argtypes = [cache, vp, i64, i64, i64, vp, i64, i64, i64, vp, vp, i32, i32, i32, f32, f32, vp, i64, vp]
    lib.dbsp_cache_attn_fwd.restype = C.c_int
    lib.dbsp_cache_attn_workspace.argtypes = [cache, i32, i32, i32, i32, i64p]
    lib.dbsp_cache_attn_workspace.restype = C.c_int
    lib.dbsp_cache_attn_layout.argtypes = [cache, i32, i32, i32, i32, C.POINTER(CacheLayout)]
    lib.dbsp_cache_attn_layout.restype = C.c_int
    lib.dbsp_cache_evict.argtypes = [cache, i32, i32, vp, vp, i64, vp]
    lib.dbsp_cache_evict.restype = C.c_int
    lib.dbsp_cache_evict_workspace.argtypes = [cache, i32, i64p]
    lib.dbsp_cache_evict_workspace.restype = C.c_int
    norm, rotary, paged, packed = C.POINTER(HeadNormDesc), C.POINTER(RotaryDesc), C.POINTER(PagedCacheDesc), C.c_char_p
    lib.dbsp_qk_norm_rope_fwd.argtypes = [packed, norm, rotary, vp]
    lib.dbsp_qk_norm_rope_fwd.restype = C.c_int
    lib.dbsp_qk_norm_rope_bwd.argtypes = [packed, packed, packed, norm, rotary, vp, vp, i64, vp]
    lib.dbsp_qk_norm_rope_bwd.restype = C.c_int
    lib.dbsp_qk_norm_rope_bwd_workspace.argtypes = [i32] * 5 + [i64p]
    lib.dbsp_qk_norm_rope_bwd_workspace.restype = C.c_int
    lib.dbsp_paged_append.argtypes = [paged, packed, packed, vp, norm, rotary, vp]
    lib.dbsp_paged_append.restype = C.c_int
    lib.dbsp_paged_attn_fwd.argtypes = [paged] + [vp, i64, i64, i64] * 2 + [vp, vp, i32, i32, i32, f32, vp, i64, vp]
    lib.dbsp_paged_attn_fwd.restype = C.c_int
    lib.dbsp_paged_attn_workspace.argtypes = [paged, i32, i32, i64p]
    lib.dbsp_paged_attn_workspace.restype = C.c_int
    lib.dbsp_plan_destroy.argtypes = [vp]
    lib.dbsp_plan_destroy.restype = None
    lib.dbsp_plan_release.argtypes = [vp]
    lib.dbsp_plan_release.restype = None
    lib.dbsp_last_error.argtypes = []
    lib.dbsp_last_error.restype = C.c_char_p
    _lib = lib
    return lib


def _check(rc: int):
    if rc != DBSP_OK:
        raise DbspError(rc, load_library().dbsp_last_error().decode("utf-8", "replace"))


class Plan:
    """Owner of a dbsp_plan*.  close() destroys it and waits for its last forward call; an object that is
    dropped without it (a step's plan that the next one replaces) is released and waits for nothing."""

    def __init__(self, handle: int, H: int, nQ: int, nK: int, block: int, pair_rows: bool = False):
        self._h = C.c_void_p(handle)
        self.H, self.nQ, self.nK, self.block = H, nQ, nK, block      # nQ, nK: the mask's block grid
        self.pair_rows = pair_rows

    @property
    def handle(self):
        if not self._h:
            raise ValueError("plan already destroyed")
        return self._h

    def array(self, what: int) -> np.ndarray:
        """Copy of one plan array (see dbsp_plan_array in dbsp.h)."""
        data, count = C.c_void_p(), C.c_int64()
        _check(load_library().dbsp_plan_get(self.handle, what, C.byref(data), C.byref(count)))
        dt = np.int64 if what in _INT64_ARRAYS else np.int32
        if count.value == 0:
            return np.zeros(0, dtype=dt)
        ctype = C.c_int64 if dt is np.int64 else C.c_int32
        buf = C.cast(data, C.POINTER(ctype * count.value)).contents
        return np.frombuffer(buf, dtype=dt).copy()

    def stats(self, with_rho: bool = True) -> dict:
        """dbsp_plan_stats.  with_rho=False leaves out rho_naive / rho_balanced (the library works those
        out on request: each costs a placement pass unless it is the placement the plan uses)."""
        rn, rb, rp, pu = C.c_double(), C.c_double(), C.c_double(), C.c_double()
        nnz, ni = C.c_int64(), C.c_int64()
        P, L = C.c_int32(), C.c_int32()
        _check(load_library().dbsp_plan_stats(self.handle, C.byref(rn) if with_rho else None, C.byref(rb) if with_rho else None,
                                              C.byref(rp), C.byref(nnz), C.byref(ni), C.byref(P), C.byref(L), C.byref(pu)))
        out = dict(rho_plan=rp.value, nnz=nnz.value, n_items=ni.value, num_partitions=P.value, max_item_len=L.value, plan_usec=pu.value)
        if with_rho:
            out.update(rho_naive=rn.value, rho_balanced=rb.value)
        return out

    def busy(self, stream=None):
        """(busy ticks uint64 [P] at 100 MHz, hw ids uint32 [P]) of the last forward call; synchronises."""
        P = self.stats(with_rho=False)["num_partitions"]
        ticks = np.zeros(P, dtype=np.uint64)
        hw = np.zeros(P, dtype=np.uint32)
        _check(load_library().dbsp_plan_busy(self.handle, ticks.ctypes.data_as(C.c_void_p),
                                             hw.ctypes.data_as(C.c_void_p), _stream_ptr(stream)))
        return ticks, hw

    def tail_takes(self, stream=None):
        """How often each item of the shared queue was taken since the plan was made (uint32 [n_tail]); synchronises."""
        n = int(self.array(TAIL_ITEMS).shape[0])
        takes = np.zeros(n, dtype=np.uint32)
        _check(load_library().dbsp_plan_tail_takes(self.handle, takes.ctypes.data_as(C.c_void_p), _stream_ptr(stream)))
        return takes

    def calibrate(self, stream=None):
        """Relative time per block of the compute units in the last forward call (int32 [P], mean about 1024):
        pass it as partition_cost to later plans with the same mode and partition count.  Synchronises."""
        cost = np.zeros(self.stats(with_rho=False)["num_partitions"], dtype=np.int32)
        _check(load_library().dbsp_plan_calibrate(self.handle, cost.ctypes.data_as(C.c_void_p), _stream_ptr(stream)))
        return cost

    def run_order(self) -> dict:
        """dbsp_plan_run_order (see dbsp_diag.h): partition_of (int32, of every workgroup), items (int32, workgroup by
        workgroup in the order they run), local, staged."""
        part = np.zeros(self.stats(with_rho=False)["num_partitions"], dtype=np.int32)
        items = np.zeros(self.array(PART_ITEMS).shape[0], dtype=np.int32)
        local, staged = C.c_int32(), C.c_int32()
        _check(load_library().dbsp_plan_run_order(self.handle, _addr(part), _addr(items), C.byref(local), C.byref(staged)))
        return dict(partition_of=part, items=items, local=bool(local.value), staged=bool(staged.value))

    def close(self):
        if self._h:
            load_library().dbsp_plan_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            if self._h:
                load_library().dbsp_plan_release(self._h)
                self._h = C.c_void_p()
        except Exception:
            pass


def plan_sparse_attn(mask, block: int, num_partitions: int = 0, mode: int = MODE_BALANCED,
                     max_item_len: int = 0, item_overhead: int = 0, host_only: bool = False,
                     locality_groups: int = 0, partition_cost=None, max_batch: int = 0, dynamic_tail: int = 0,
                     reward: float = 0.0, pair_rows: bool = False, head_dim: int = 0) -> Plan:
    """mask: uint8 host array [H, nQ, nK]; returns a Plan (see dbsp.h: plan_sparse_attn)."""
    mask = np.ascontiguousarray(mask, dtype=np.uint8)
    if mask.ndim != 3:
        raise ValueError("mask must be [H, nQ, nK]")
    H, nQ, nK = mask.shape
    cost = np.ascontiguousarray(partition_cost, dtype=np.int32) if partition_cost is not None else None
    if cost is not None:
        if num_partitions == 0:
            num_partitions = int(cost.shape[0])      # one cost per partition: the array fixes their number
        if cost.ndim != 1 or cost.shape[0] != num_partitions:
            raise ValueError("partition_cost must hold one value per partition")
    if pair_rows not in (False, True, "auto"):
        raise ValueError('pair_rows is False, True or "auto"')
    flags = (PLAN_HOST_ONLY if host_only else 0) | (PLAN_PAIR_AUTO if pair_rows == "auto" else PLAN_PAIR_ROWS if pair_rows else 0)
    opts = PlanOpts(num_partitions, mode, max_item_len, item_overhead, flags, locality_groups,
                    cost.ctypes.data_as(C.c_void_p) if cost is not None else None, max_batch, dynamic_tail, float(reward),
                    head_dim)
    lib, out = load_library(), C.c_void_p()
    rc = lib.plan_sparse_attn(_addr(mask), H, nQ, nK, block, C.byref(opts), C.byref(out))
    if rc:
        _check(rc)
    if pair_rows == "auto":
        chosen = C.c_int32()
        _check(lib.dbsp_plan_pair_rows(out, C.byref(chosen)))
        pair_rows = bool(chosen.value)
    return Plan(out.value, H, nQ, nK, block, bool(pair_rows))


def plan_sparse_attn_reuse(previous: Plan, mask, reuse_threshold: float, num_partitions: int = 0, mode: int = MODE_BALANCED,
                           max_item_len: int = 0, item_overhead: int = 0, host_only: bool = False, locality_groups: int = 0,
                           partition_cost=None, max_batch: int = 0, dynamic_tail: int = 0):
    """Plan the next mask of a sequence, keeping `previous`'s placement while rho_s under it stays
    <= reuse_threshold (see dbsp.h: plan_sparse_attn_reuse).  Returns (Plan, reused, rho_under_previous)."""
    mask = np.ascontiguousarray(mask, dtype=np.uint8)
    if mask.shape != (previous.H, previous.nQ, previous.nK):
        raise ValueError("mask shape differs from the previous plan's")
    cost = np.ascontiguousarray(partition_cost, dtype=np.int32) if partition_cost is not None else None
    if cost is not None:
        if num_partitions == 0:
            num_partitions = int(cost.shape[0])      # one cost per partition: the array fixes their number
        if cost.ndim != 1 or cost.shape[0] != num_partitions:
            raise ValueError("partition_cost must hold one value per partition")
    flags = (PLAN_HOST_ONLY if host_only else 0) | (PLAN_PAIR_ROWS if previous.pair_rows else 0)   # pair rows are kept
    opts = PlanOpts(num_partitions, mode, max_item_len, item_overhead, flags, locality_groups,
                    cost.ctypes.data_as(C.c_void_p) if cost is not None else None, max_batch, dynamic_tail, 0.0)
    out, reused, rho = C.c_void_p(), C.c_int32(), C.c_double()
    _check(load_library().plan_sparse_attn_reuse(previous.handle, _addr(mask), C.byref(opts),
                                                 float(reuse_threshold), C.byref(out), C.byref(reused), C.byref(rho)))
    return (Plan(out.value, previous.H, previous.nQ, previous.nK, previous.block, previous.pair_rows),
            bool(reused.value), rho.value)


def _addr(array) -> int:
    """Address of a numpy array's data (ndarray.ctypes builds an object per call)."""
    return array.__array_interface__["data"][0]


def _stream_ptr(stream):
    if stream is None:
        import torch
        if torch.cuda.is_available():
            return C.c_void_p(torch.cuda.current_stream().cuda_stream)
        return C.c_void_p(0)
    if isinstance(stream, int):
        return C.c_void_p(stream)
    return C.c_void_p(stream.cuda_stream)


def sparse_attn_fwd(plan: Plan, q, k, v, o=None, lse=None, softmax_scale: float = 0.0, stream=None, want_lse: bool = True,
                    static_scratch: bool = False):
    """q [B,H,Nq,d], k/v [B,H,Nk,d]: contiguous bf16 torch tensors on the GPU.  Enqueues on
    `stream` (default: torch's current stream) and returns (o, lse) without synchronising.
    static_scratch=True calls sparse_attn_fwd_static (pass o and lse then: this wrapper allocates
    the ones it is not given)."""
    global _torch
    if _torch is None:
        import torch as _torch_module
        _torch = _torch_module
    torch = _torch
    bf16 = torch.bfloat16
    if not (q.dtype == k.dtype == v.dtype == bf16 and q.is_cuda and k.is_cuda and v.is_cuda
            and q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and q.dim() == k.dim() == v.dim() == 4):
        for name, x in (("q", q), ("k", k), ("v", v)):
            if x.dtype != bf16 or not x.is_cuda or not x.is_contiguous() or x.dim() != 4:
                raise ValueError(f"{name} must be a contiguous 4-d bf16 tensor on the GPU")
    B, H, Nq, d = q.shape
    kshape = k.shape
    Nk = kshape[2]
    if kshape != (B, H, Nk, d) or v.shape != kshape or H != plan.H:
        raise ValueError("q/k/v shapes disagree with each other or with the plan")
    if o is None:
        o = torch.empty_like(q)
    if lse is None and want_lse:
        lse = q.new_empty((B, H, Nq), dtype=torch.float32)
    if stream is None:
        # the raw handle of torch's current stream, as a kernel launch needs it
        stream = torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    lib = load_library()
    entry = lib.sparse_attn_fwd_static if static_scratch else lib.sparse_attn_fwd
    rc = entry(plan.handle, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), None if lse is None else lse.data_ptr(),
               B, Nq, Nk, d, float(softmax_scale), stream)
    if rc:
        _check(rc)
    return o, lse


def _torch_module():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


class _OnDevice:
    """What has tensors on a GPU (device, _index) and is called on streams."""

    def _on(self, stream):
        """The raw stream, and whether tensors made on torch's current one are used on another."""
        torch = _torch
        if self._index != torch._C._cuda_getDevice():
            raise ValueError("the tensors live on another device than the current one")
        now = torch._C._cuda_getCurrentRawStream(self._index)
        if stream is None:
            return now, False
        if isinstance(stream, int):
            return stream, stream != now
        if getattr(stream, "device", self.device) != self.device:
            raise ValueError("the stream is of another device than the tensors")
        raw = stream.cuda_stream
        return raw, raw != now

    def _empty(self, shape, dtype, raw, elsewhere):
        """A tensor for a call on the stream raw.  Memory that torch's current stream has freed may still be used there, so for a call
        elsewhere it comes from that stream's; freed, it waits for what the current stream has been given until then."""
        torch = _torch
        if not elsewhere:
            return torch.empty(shape, dtype=dtype, device=self.device)
        # (an ExternalStream of handle 0 would be some stream of torch's pool, not the default stream)
        on = torch.cuda.ExternalStream(raw, device=self.device) if raw else torch.cuda.default_stream(self.device)
        with torch.cuda.stream(on):
            x = torch.empty(shape, dtype=dtype, device=self.device)
        x.record_stream(torch.cuda.current_stream(self.device))
        return x

    def _workspace(self, workspace, key, ask, raw, elsewhere):
        """The caller's workspace, or one of the size that a call with these sizes (key) needs; its address and size."""
        torch = _torch
        if workspace is None:
            need = self._bytes.get(key)
            if need is None:
                out = C.c_int64()
                _check(ask(self._at, *key, C.byref(out)))
                need = self._bytes[key] = out.value
            if need == 0:
                return None, None, 0
            workspace = self._empty(need, torch.uint8, raw, elsewhere)
        elif workspace.dtype != torch.uint8 or workspace.device != self.device or not workspace.is_contiguous():
            raise ValueError("the workspace must be a contiguous uint8 tensor on the cache's GPU")
        return workspace, workspace.data_ptr(), workspace.numel()


class _Kept:
    """What keeps tensors of the caller and describes them to the library by their addresses.  A tensor may be given other memory (x.data = y, as a
    module's half() and to() do with its parameters; resize_()): then its address is another one, as what is described is held until the next call."""

    def _keep(self, *tensors):
        self._described = tuple((x.data_ptr, x.data_ptr()) for x in tensors)
        self._held = tuple(x.detach() for x in tensors)

    def _now(self):
        """Describes the tensors anew, and checks them again, where one of them has been given other memory."""
        for address, was in self._described:
            if address() != was:
                self._again()
                break


class KVCache(_OnDevice, _Kept):
    """A key/value cache of the caller's tensors (see dbsp.h: dbsp_cache), for cache_attn_fwd and cache_evict.

    k, v: [B, Hk, capacity, d], bf16 or fp16 on one GPU, d in (64, 128) dense, other strides multiples of 8 elements; the first
    lens[b] (int32 [B] there) slots of sequence b are used.  prefix_k, prefix_v: [Hk, P, d], shared by all sequences.  Either
    pair may be missing.  weights: f32 [B, Hk, capacity], positions: int32 [B, Hk, capacity], both contiguous.  The object keeps the
    tensors, which the caller goes on writing, and every call goes by the memory that they have then (what they had before is held until that call);
    it copies nothing, and other tensors make another object."""

    def __init__(self, k=None, v=None, lens=None, prefix_k=None, prefix_v=None, weights=None, positions=None):
        torch = _torch_module()
        load_library()
        some = k if k is not None else prefix_k
        if some is None or (k is None) != (v is None) or (prefix_k is None) != (prefix_v is None) or (k is None) != (lens is None):
            raise ValueError("a cache has k, v and lens, or prefix_k and prefix_v, or all of them")
        if some.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("keys and values are bf16 or fp16")
        self.dtype, self.device, d = some.dtype, some.device, some.shape[-1]
        desc = CacheDesc(dtype=0 if some.dtype == torch.bfloat16 else 1, d=d)
        for name, x, dims in (("k", k, 4), ("v", v, 4), ("prefix_k", prefix_k, 3), ("prefix_v", prefix_v, 3)):
            if x is None:
                continue
            if x.dim() != dims or x.dtype != self.dtype or not x.is_cuda or x.device != self.device or x.shape[-1] != d or x.stride(-1) != 1:
                raise ValueError(f"{name} must be a {dims}-d tensor of the cache's type and head dim on its GPU, with a dense last dimension")
            setattr(desc, name, x.data_ptr())
            stride = getattr(desc, name + "_stride")
            for i in range(dims - 1):
                stride[i] = x.stride(i)
        if k is not None:
            if k.shape != v.shape:
                raise ValueError("k and v differ in shape")
            desc.B, desc.Hk, desc.capacity = k.shape[:3]
        if prefix_k is not None:
            if prefix_k.shape != prefix_v.shape or (k is not None and prefix_k.shape[0] != k.shape[1]):
                raise ValueError("prefix_k and prefix_v differ in shape, or from k in their heads")
            desc.Hk, desc.n_prefix = prefix_k.shape[:2]
        for name, x, dtype, shape in (("lens", lens, torch.int32, k.shape[:1] if k is not None else None),
                                      ("weights", weights, torch.float32, k.shape[:3] if k is not None else None),
                                      ("positions", positions, torch.int32, k.shape[:3] if k is not None else None)):
            if x is None:
                continue
            if shape is None or x.dtype != dtype or x.device != self.device or x.shape != shape or not x.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {dtype} tensor of {'[B]' if name == 'lens' else '[B, Hk, capacity]'} on the cache's GPU")
            setattr(desc, name, x.data_ptr())
        self.k, self.v, self.lens, self.prefix_k, self.prefix_v, self.weights, self.positions = k, v, lens, prefix_k, prefix_v, weights, positions
        self.B, self.Hk, self.d, self.capacity, self.n_prefix = desc.B if k is not None else None, desc.Hk, d, desc.capacity, desc.n_prefix
        self._desc, self._at, self._bytes, self._index = desc, C.byref(desc), {}, some.get_device()
        self._keep(*(x for x in (k, v, lens, prefix_k, prefix_v, weights, positions) if x is not None))

    def _again(self):
        self.__init__(self.k, self.v, self.lens, self.prefix_k, self.prefix_v, self.weights, self.positions)

    def _for(self, B):
        """The same prefix for B sequences."""
        other = copy.copy(self)
        other._desc = CacheDesc.from_buffer_copy(self._desc)
        other._desc.B = other.B = B
        other._at, other._bytes = C.byref(other._desc), {}
        return other


def cache_attn_fwd(cache: KVCache, q, q_lens=None, causal: bool = True, decay=None, o=None, lse=None, softmax_scale: float = 0.0,
                   stream=None, want_lse: bool = True, workspace=None):
    """Attention of each sequence's newest tokens, q [B, H, Nq, d], over the cache's shared prefix and its own keys (see dbsp.h:
    dbsp_cache_attn_fwd; the new tokens' keys are written before).  q_lens: int32 [B] on the GPU, if not all Nq tokens are there;
    the others' rows of o and lse are left as they were, so pass o and lse then.  decay: None, or the factor of what the cache's
    weights hold, to which this call's attention is added.  Enqueues on `stream` (default: torch's current stream) and
    returns (o, lse)."""
    torch = _torch
    cache._now()
    shape, q_s = q.shape, q.stride()
    if len(shape) != 4 or q.dtype != cache.dtype or q.device != cache.device or shape[3] != cache.d or q_s[3] != 1:
        raise ValueError("q must be [B, H, Nq, d] of the cache's type and head dim on its GPU, with a dense last dimension")
    B, H, Nq, _ = shape
    if cache.B is None:
        cache = cache._for(B)                        # a prefix alone serves any number of sequences
    elif B != cache.B:
        raise ValueError("q and the cache differ in the number of sequences")
    raw, elsewhere = cache._on(stream)
    if o is None:
        o = cache._empty(shape, q.dtype, raw, elsewhere)
    elif o.shape != shape or o.dtype != q.dtype or o.device != q.device or o.stride(3) != 1:
        raise ValueError("o must be as q")
    if lse is None:
        if want_lse:
            lse = cache._empty((B, H, Nq), torch.float32, raw, elsewhere)
    elif lse.shape != (B, H, Nq) or lse.dtype != torch.float32 or lse.device != q.device or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous f32 tensor of [B, H, Nq] on q's GPU")
    if q_lens is not None and (q_lens.shape != (B,) or q_lens.dtype != torch.int32 or q_lens.device != q.device or not q_lens.is_contiguous()):
        raise ValueError("q_lens must be a contiguous int32 tensor of [B] on q's GPU")
    if decay is None:
        decay = -1.0
    elif not decay >= 0:
        raise ValueError("decay must not be negative")
    elif cache.weights is None:
        raise ValueError("the cache has no weights")
    lib = _lib
    workspace, at, size = cache._workspace(workspace, (H, Nq, causal, decay >= 0), lib.dbsp_cache_attn_workspace, raw, elsewhere)
    o_s = o.stride()
    rc = lib.dbsp_cache_attn_fwd(cache._at, q.data_ptr(), q_s[0], q_s[1], q_s[2], o.data_ptr(), o_s[0], o_s[1], o_s[2], None if lse is None else lse.data_ptr(),
                                 None if q_lens is None else q_lens.data_ptr(), H, Nq, causal, softmax_scale, decay, at, size, raw)
    if rc:
        _check(rc)
    return o, lse


def cache_evict(cache: KVCache, budget: int, sinks: int = 0, keep_from=None, stream=None, workspace=None) -> None:
    """Cuts the sequences with more than `budget` used slots back to the `budget` keys of the largest weights, in place, each KV
    head by itself (see dbsp.h: dbsp_cache_evict).  Keys at positions below `sinks`, and from keep_from[b] on (int32 [B] on the
    GPU), rank above all others.  Updates k, v, weights, positions and lens; enqueues on `stream`."""
    if cache.k is None:
        raise ValueError("the cache has no keys of its own")
    torch = _torch
    cache._now()
    raw, elsewhere = cache._on(stream)
    if keep_from is not None and (keep_from.shape != (cache.B,) or keep_from.dtype != torch.int32 or keep_from.device != cache.device or not keep_from.is_contiguous()):
        raise ValueError("keep_from must be a contiguous int32 tensor of [B] on the cache's GPU")
    workspace, at, size = cache._workspace(workspace, (budget,), _lib.dbsp_cache_evict_workspace, raw, elsewhere)
    rc = _lib.dbsp_cache_evict(cache._at, budget, sinks, None if keep_from is None else keep_from.data_ptr(), at, size, raw)
    if rc:
        _check(rc)


_NORMS = {"rms": 1, "layer": 2}


class HeadNorm(_Kept):
    """The norm of each head of queries and keys by itself (see dbsp.h: dbsp_head_norm; not that of all heads of a token together, with a gain of
    [H d], which some models have): kind "rms" or "layer"; gains and biases are [d] tensors on the GPU, all f32 or all of the rows' type, and a missing one is 1 or 0.  The object keeps the tensors, which the caller goes on writing, and every call
    goes by the memory that they have then."""

    def __init__(self, q_gain=None, k_gain=None, q_bias=None, k_bias=None, kind: str = "rms", eps: float = 1e-6):
        torch = _torch_module()
        load_library()
        if kind not in _NORMS:
            raise ValueError('kind is "rms" or "layer"')
        self.given = {name: x for name, x in (("q_gain", q_gain), ("k_gain", k_gain), ("q_bias", q_bias), ("k_bias", k_bias)) if x is not None}
        self.kind, self.eps, self.dtype, self.device, self.d = kind, float(eps), None, None, None
        desc = HeadNormDesc(kind=_NORMS[kind], eps=self.eps)
        for name, x in self.given.items():
            if x.dtype not in (torch.float32, torch.bfloat16, torch.float16) or x.dim() != 1 or not x.is_cuda or not x.is_contiguous():
                raise ValueError(f"{name} must be a contiguous [d] tensor of f32, bf16 or fp16 on the GPU")
            if self.dtype is not None and (x.dtype != self.dtype or x.device != self.device or x.shape[0] != self.d):
                raise ValueError("gains and biases differ in type, device or size")
            if not x.data_ptr():
                raise ValueError(f"{name} has no memory")
            self.dtype, self.device, self.d = x.dtype, x.device, x.shape[0]
            setattr(desc, name, x.data_ptr())
        self._wide, self._index = self.dtype is torch.float32, None if self.device is None else x.get_device()
        desc.gains_f32 = self._wide
        self._desc, self._at = desc, C.byref(desc)
        self._keep(*self.given.values())

    def _again(self):
        self.__init__(**self.given, kind=self.kind, eps=self.eps)

    def _of(self, x):
        """What a call on tensors like x passes on."""
        self._now()
        if self.d is not None and (self._index != x.get_device() or self.d != x.shape[-1] or not (self._wide or self.dtype is x.dtype)):
            raise ValueError("gains and biases must be [d], f32 or of the rows' type, on their GPU")
        return self._at


class Rotary:
    """A rotation by positions on one to four axes (see dbsp.h: dbsp_rotary).  pairs: how many pairs of a head each axis turns; pair i of an
    axis with n of them by theta^(-i / n) a unit, or freqs says so for all pairs, axis by axis.  halves: a pair's two places are R apart (R all
    pairs) instead of neighbours."""

    def __init__(self, pairs, theta: float = 10000.0, halves: bool = False, freqs=None):
        load_library()
        self.pairs = tuple(int(n) for n in pairs)
        if not 1 <= len(self.pairs) <= 4 or min(self.pairs) < 1:
            raise ValueError("a rotation has one to four axes of at least one pair each")
        self.halves = bool(halves)
        self.freqs = tuple(float(f) for f in freqs) if freqs is not None else tuple(float(theta) ** (-i / n) for n in self.pairs for i in range(n))
        if len(self.freqs) != sum(self.pairs):
            raise ValueError("freqs must hold one value per pair")
        self._freqs = (C.c_double * len(self.freqs))(*self.freqs)
        self.axes = len(self.pairs)
        desc = RotaryDesc(axes=self.axes, halves=self.halves, freqs=self._freqs)
        desc.pairs[:len(self.pairs)] = self.pairs
        self._desc, self._at = desc, C.byref(desc)


class _Rows(_OnDevice):
    """Where calls on rows of a GPU run, and the sizes of workspaces that they have asked for."""

    def __init__(self, index):
        self.device, self._index, self._at, self._bytes = _torch.device("cuda", index), index, None, {}


_rows_on, _ROW_TYPES = {}, {}


def _on_rows(q):
    """What q's calls run on; q is a tensor that they can begin with."""
    here = _rows_on.get(q.get_device())
    if here is None:
        torch = _torch_module()
        if not q.is_cuda:
            raise ValueError("q must be on a GPU")
        load_library()
        _ROW_TYPES.update({torch.bfloat16: 0, torch.float16: 1})
        here = _rows_on[q.get_device()] = _Rows(q.get_device())
    if q.dim() != 4 or q.dtype not in _ROW_TYPES:
        raise ValueError("q must be [B, H, N, d] in bf16 or fp16")
    return here


def _heads(name, x, shape, dtype, index):
    """Address and strides (batch, head, token) of rows."""
    s = x.stride()
    if x.shape != shape or x.dtype is not dtype or x.get_device() != index or s[3] != 1:
        raise ValueError(f"{name} must be {list(shape)} of the same type on the same GPU, with a dense last dimension")
    return x.data_ptr(), s[0], s[1], s[2]


def _positions(positions, rotary, B, N, index):
    """Address and strides (batch, token) of positions [N, axes] or [B, N, axes]."""
    if positions is None or rotary is None:
        return _NO_POSITIONS
    shape, s = positions.shape, positions.stride()
    tokens = shape == (N, rotary.axes)
    if not (tokens or shape == (B, N, rotary.axes)) or positions.dtype is not _torch.int32 or positions.get_device() != index or (s[-1] != 1 and rotary.axes > 1):
        raise ValueError("positions must be int32 [N, axes] or [B, N, axes] on the same GPU, with a dense last dimension")
    return positions.data_ptr(), 0 if tokens else s[0], s[-2]


def qk_norm_rope_fwd(q, k=None, norm: HeadNorm = None, rotary: Rotary = None, positions=None, q_out=None, k_out=None, stream=None):
    """Queries [B, H, N, d] and keys [B, Hk, N, d] of a projection (any strides: views into its output) with each head's norm and the rotation
    by positions (int32 [N, axes] or [B, N, axes]; None with one axis: 0 .. N - 1), as contiguous tensors or in q_out and k_out
    (see dbsp.h: dbsp_qk_norm_rope_fwd).  Autograd does not see the call: gradients are qk_norm_rope_bwd's.  Enqueues on `stream` (default: torch's current stream) and returns (q_out, k_out)."""
    here = _on_rows(q)
    raw, elsewhere = here._on(stream)
    shape, dtype, index = q.shape, q.dtype, here._index
    B, H, N, d = shape
    if q_out is None:
        q_out = here._empty(shape, dtype, raw, elsewhere)
    Hk, k_at, k_out_at = 0, _NO_HEADS, _NO_HEADS
    if k is not None:
        if k.dim() == 4:
            Hk = k.shape[1]
        shape_k = (B, Hk, N, d)
        k_at = _heads("k", k, shape_k, dtype, index)
        if k_out is None:
            k_out = here._empty(shape_k, dtype, raw, elsewhere)
        k_out_at = _heads("k_out", k_out, shape_k, dtype, index)
    elif k_out is not None:
        raise ValueError("k_out without k")
    rows = _QK_ROWS.pack(_ROW_TYPES[dtype], B, N, d, H, Hk, *_heads("q", q, shape, dtype, index), *k_at, *_heads("q_out", q_out, shape, dtype, index),
                         *k_out_at, *_positions(positions, rotary, B, N, index))
    rc = _lib.dbsp_qk_norm_rope_fwd(rows, None if norm is None else norm._of(q), None if rotary is None else rotary._at, raw)
    if rc:
        _check(rc)
    return q_out, k_out


_GAINS = ("q_gain", "k_gain", "q_bias", "k_bias")


def qk_norm_rope_bwd(q, k, dq_out, dk_out, norm: HeadNorm = None, rotary: Rotary = None, positions=None, dq=None, dk=None, stream=None, workspace=None):
    """Gradients of a qk_norm_rope_fwd call: from its q, k (or None), norm, rotary and positions and the gradients of its results, those of q and k
    (contiguous tensors, or dq and dk, which may be views into the gradient of a projection's output), and of the gains and biases that the
    norm has, f32 [d] by name (see dbsp.h: dbsp_qk_norm_rope_bwd).  Enqueues on `stream` and returns (dq, dk, gains)."""
    here = _on_rows(q)
    raw, elsewhere = here._on(stream)
    shape, dtype, index = q.shape, q.dtype, here._index
    B, H, N, d = shape
    if dq is None:
        dq = here._empty(shape, dtype, raw, elsewhere)
    Hk, k_at, k_out_at, dk_at = 0, _NO_HEADS, _NO_HEADS, None
    if k is not None:
        if k.dim() == 4:
            Hk = k.shape[1]
        shape_k = (B, Hk, N, d)
        k_at = _heads("k", k, shape_k, dtype, index)
        if dk_out is None:
            raise ValueError("k without dk_out")
        k_out_at = _heads("dk_out", dk_out, shape_k, dtype, index)
        if dk is None:
            dk = here._empty(shape_k, dtype, raw, elsewhere)
        dk_at = _HEADS.pack(*_heads("dk", dk, shape_k, dtype, index))
    elif dk_out is not None or dk is not None:
        raise ValueError("dk_out or dk without k")
    rows = _QK_ROWS.pack(_ROW_TYPES[dtype], B, N, d, H, Hk, *_heads("q", q, shape, dtype, index), *k_at, *_heads("dq_out", dq_out, shape, dtype, index),
                         *k_out_at, *_positions(positions, rotary, B, N, index))
    dq_at = _HEADS.pack(*_heads("dq", dq, shape, dtype, index))
    norm_at, grads, grads_at, at, size, gains = None, None, None, None, 0, {}
    if norm is not None:
        norm_at = norm._of(q)
        if norm.given:
            grads = here._empty((4, d), _torch.float32, raw, elsewhere)
            grads_at = grads.data_ptr()
            if len(here._bytes) > 1000:              # (a program whose sizes never come back)
                here._bytes.clear()
            workspace, at, size = here._workspace(workspace, (B, N, d, H, Hk), _grads_workspace, raw, elsewhere)
    rc = _lib.dbsp_qk_norm_rope_bwd(rows, dq_at, dk_at, norm_at, None if rotary is None else rotary._at, grads_at, at, size, raw)
    if rc:
        _check(rc)
    if grads is not None:
        gains = {name: x for name, x in zip(_GAINS, grads.unbind()) if name in norm.given and (k is not None or name[0] == "q")}
    return dq, dk, gains


def _grads_workspace(_, *sizes):
    return _lib.dbsp_qk_norm_rope_bwd_workspace(*sizes)


class PagedKVCache(_OnDevice, _Kept):
    """A key/value cache in pages of the caller's tensors (see dbsp.h: dbsp_paged_cache), for paged_append and paged_attn_fwd.

    k, v: the pool, [n_pages, Hk, page_size, d], bf16 or fp16 on one GPU, d in (64, 128) dense, other strides multiples of 8 elements (a pool of
    [n_pages, page_size, Hk, d] goes in as its transpose(1, 2)).  pages: int32 [B, max_pages], the pages of each sequence's slots, an entry that
    is no page where a sequence has none.  lens: int32 [B], used slots.  The object keeps the tensors, which the caller goes on writing, and
    every call goes by the memory that they have then (what they had before is held until that call); other tensors make another object."""

    def __init__(self, k, v, pages, lens):
        torch = _torch_module()
        load_library()
        if k.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("keys and values are bf16 or fp16")
        for name, x in (("k", k), ("v", v)):
            if x.dim() != 4 or x.dtype != k.dtype or not x.is_cuda or x.device != k.device or x.shape != k.shape or x.stride(3) != 1:
                raise ValueError(f"{name} must be a tensor of [n_pages, Hk, page_size, d] on the cache's GPU, with a dense last dimension")
        if pages.dim() != 2 or pages.dtype != torch.int32 or pages.device != k.device or (pages.shape[1] > 1 and pages.stride(1) != 1):
            raise ValueError("pages must be int32 [B, max_pages] on the cache's GPU, with a dense last dimension")
        if lens.shape != pages.shape[:1] or lens.dtype != torch.int32 or lens.device != k.device or not lens.is_contiguous():
            raise ValueError("lens must be a contiguous int32 tensor of [B] on the cache's GPU")
        self.k, self.v, self.pages, self.lens = k, v, pages, lens
        self.dtype, self.device, self._index = k.dtype, k.device, k.get_device()
        self.B, self.max_pages = pages.shape
        self.n_pages, self.Hk, self.page_size, self.d = k.shape
        desc = PagedCacheDesc(dtype=k.dtype == torch.float16, B=self.B, Hk=self.Hk, d=self.d, n_pages=self.n_pages, page_size=self.page_size,
                              max_pages=self.max_pages, k=k.data_ptr(), v=v.data_ptr(), pages=pages.data_ptr(), pages_stride=pages.stride(0), lens=lens.data_ptr())
        desc.k_stride[:], desc.v_stride[:] = k.stride()[:3], v.stride()[:3]
        self._desc, self._at, self._bytes = desc, C.byref(desc), {}
        self._keep(k, v, pages, lens)

    def _again(self):
        self.__init__(self.k, self.v, self.pages, self.lens)


def paged_append(cache: PagedKVCache, k, v, new_lens=None, q=None, q_out=None, norm: HeadNorm = None, rotary: Rotary = None, positions=None, stream=None):
    """Writes the keys and values [B, Hk, Nn, d] of each sequence's newest tokens into its last used slots (cache.lens counts them already), keys
    with norm and rotation on the way, and beside them the tokens' queries q [B, H, Nn, d] into q_out (see dbsp.h: dbsp_paged_append).  new_lens:
    int32 [B] on the GPU, if not all Nn tokens are there; the others' rows of q_out are left as they were, so pass it then.  positions:
    int32 [Nn, axes] or [B, Nn, axes], None with one axis: the tokens' slots.  Enqueues on `stream` and returns q_out (None without q)."""
    cache._now()
    B, Hk, d, dtype, index = cache.B, cache.Hk, cache.d, cache.dtype, cache._index
    if k.dim() != 4:
        raise ValueError("k must be [B, Hk, Nn, d]")
    Nn = k.shape[2]
    shape = (B, Hk, Nn, d)
    raw, elsewhere = cache._on(stream)
    H, q_at, o_at = 0, _NO_HEADS, _NO_HEADS
    if q is not None:
        if q.dim() != 4:
            raise ValueError("q must be [B, H, Nn, d]")
        H = q.shape[1]
        shape_q = (B, H, Nn, d)
        q_at = _heads("q", q, shape_q, dtype, index)
        if q_out is None:
            q_out = cache._empty(shape_q, dtype, raw, elsewhere)
        o_at = _heads("q_out", q_out, shape_q, dtype, index)
    elif q_out is not None:
        raise ValueError("q_out without q")
    new_at = None
    if new_lens is not None:
        if new_lens.shape != (B,) or new_lens.dtype is not _torch.int32 or new_lens.get_device() != index or not new_lens.is_contiguous():
            raise ValueError("new_lens must be a contiguous int32 tensor of [B] on the cache's GPU")
        new_at = new_lens.data_ptr()
    rows = _QK_ROWS.pack(dtype is _torch.float16, B, Nn, d, H, Hk, *q_at, *_heads("k", k, shape, dtype, index), *o_at, *_NO_HEADS,
                         *_positions(positions, rotary, B, Nn, index))
    rc = _lib.dbsp_paged_append(cache._at, rows, _HEADS.pack(*_heads("v", v, shape, dtype, index)), new_at, None if norm is None else norm._of(k),
                                None if rotary is None else rotary._at, raw)
    if rc:
        _check(rc)
    return q_out


def paged_attn_fwd(cache: PagedKVCache, q, q_lens=None, causal: bool = True, o=None, lse=None, softmax_scale: float = 0.0, stream=None, want_lse: bool = True,
                   workspace=None):
    """Attention of each sequence's newest tokens, q [B, H, Nq, d], over its pages (see dbsp.h: dbsp_paged_attn_fwd; the new tokens' keys are written
    before).  q_lens: int32 [B] on the GPU, if not all Nq tokens are there; the others' rows of o and lse are left as they were, so pass o
    and lse then.  Enqueues on `stream` (default: torch's current stream) and returns (o, lse)."""
    cache._now()
    shape, q_s, dtype, index = q.shape, q.stride(), cache.dtype, cache._index
    if len(shape) != 4 or q.dtype is not dtype or q.get_device() != index or shape[0] != cache.B or shape[3] != cache.d or q_s[3] != 1:
        raise ValueError("q must be [B, H, Nq, d] of the cache's sequences, type and head dim on its GPU, with a dense last dimension")
    B, H, Nq, _ = shape
    raw, elsewhere = cache._on(stream)
    if o is None:
        o = cache._empty(shape, dtype, raw, elsewhere)
    o_at, *o_s = _heads("o", o, shape, dtype, index)
    if lse is None:
        if want_lse:
            lse = cache._empty((B, H, Nq), _torch.float32, raw, elsewhere)
    elif lse.shape != (B, H, Nq) or lse.dtype is not _torch.float32 or lse.get_device() != index or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous f32 tensor of [B, H, Nq] on q's GPU")
    if q_lens is not None and (q_lens.shape != (B,) or q_lens.dtype is not _torch.int32 or q_lens.get_device() != index or not q_lens.is_contiguous()):
        raise ValueError("q_lens must be a contiguous int32 tensor of [B] on q's GPU")
    lib = _lib
    workspace, at, size = cache._workspace(workspace, (H, Nq), lib.dbsp_paged_attn_workspace, raw, elsewhere)
    rc = lib.dbsp_paged_attn_fwd(cache._at, q.data_ptr(), q_s[0], q_s[1], q_s[2], o_at, *o_s, None if lse is None else lse.data_ptr(),
                                 None if q_lens is None else q_lens.data_ptr(), H, Nq, causal, softmax_scale, at, size, raw)
    if rc:
        _check(rc)
    return o, lse


def imbalance_ratio(work) -> float:
    """Eq. 1 of the paper on an integer matrix work[periods][partitions]."""
    w = np.ascontiguousarray(work, dtype=np.int64)
    if w.ndim == 1:
        w = w[None]
    rho = C.c_double()
    _check(load_library().imbalance_ratio(w.ctypes.data_as(C.c_void_p), w.shape[0], w.shape[1], C.byref(rho)))
    return rho.value


def _ptr(a):
    return _addr(a) if a is not None else None


def _split(flat, ptr):
    return [flat[ptr[g]:ptr[g + 1]].tolist() for g in range(len(ptr) - 1)]


def partition_heads(blocks_per_head, x: int, capacity: int = 0, previous=None, reuse_threshold: float = 1.0) -> dict:
    """Head-level partitioning over x GPUs with plan reuse (see dbsp.h: dbsp_partition_heads)."""
    cnt = np.ascontiguousarray(blocks_per_head, dtype=np.int64)
    H = cnt.shape[0]
    prev = np.ascontiguousarray(previous, dtype=np.int32) if previous is not None else None
    if prev is not None and prev.shape != (H,):
        raise ValueError("previous plan must hold one GPU id per head")
    where, lst, ptr = np.empty(H, np.int32), np.empty(H, np.int32), np.empty(max(x, 0) + 1, np.int32)
    load = np.empty(max(x, 0), np.int64)
    rc_, rp_, r_, reused = C.c_double(), C.c_double(), C.c_double(), C.c_int32()
    _check(load_library().dbsp_partition_heads(_ptr(cnt), H, x, capacity, _ptr(prev), float(reuse_threshold), _ptr(where), _ptr(lst),
                                               _ptr(ptr), _ptr(load), C.byref(rc_), C.byref(rp_), C.byref(r_), C.byref(reused)))
    return dict(gpu_of_head=where.tolist(), lists=_split(lst, ptr), loads=load.tolist(), rho_contiguous=rc_.value,
                rho=r_.value, rho_previous=rp_.value, reused=bool(reused.value))


def partition_blocks(mask, y: int, reward: float = 0.0, capacity_q: int = 0, capacity_kv: int = 0) -> dict:
    """Block-level partitioning of a mask [H, nQ, nK] for a ring of y GPUs (see dbsp.h: dbsp_partition_blocks)."""
    mask = np.ascontiguousarray(mask, dtype=np.uint8)
    if mask.ndim != 3:
        raise ValueError("mask must be [H, nQ, nK]")
    H, nQ, nK = mask.shape
    yy = max(y, 0)
    gq, ql, qp = np.empty(nQ, np.int32), np.empty(nQ, np.int32), np.empty(yy + 1, np.int32)
    gk, kl, kp = np.empty(nK, np.int32), np.empty(nK, np.int32), np.empty(yy + 1, np.int32)
    work = np.empty((yy, yy), np.int64)
    rc_, r_, mq, mk = C.c_double(), C.c_double(), C.c_int64(), C.c_int64()
    _check(load_library().dbsp_partition_blocks(_ptr(mask), H, nQ, nK, y, float(reward), capacity_q, capacity_kv, _ptr(gq), _ptr(ql),
                                                _ptr(qp), _ptr(gk), _ptr(kl), _ptr(kp), _ptr(work), C.byref(rc_), C.byref(r_),
                                                C.byref(mq), C.byref(mk)))
    return dict(gpu_of_q=gq.tolist(), q_lists=_split(ql, qp), chunk_of_kv=gk.tolist(), kv_lists=_split(kl, kp),
                work=work.tolist(), rho=r_.value, rho_contiguous=rc_.value, moved_q=mq.value, moved_kv=mk.value)


def ring_work(mask, y: int, gpu_of_q=None, chunk_of_kv=None):
    """Eq. 3's work matrix [iteration][GPU] and its rho_s for given maps (None = contiguous layout)."""
    mask = np.ascontiguousarray(mask, dtype=np.uint8)
    H, nQ, nK = mask.shape
    gq = np.ascontiguousarray(gpu_of_q, dtype=np.int32) if gpu_of_q is not None else None
    gk = np.ascontiguousarray(chunk_of_kv, dtype=np.int32) if chunk_of_kv is not None else None
    if (gq is not None and gq.shape != (nQ,)) or (gk is not None and gk.shape != (nK,)):
        raise ValueError("maps must hold one id per block")
    work = np.empty((max(y, 0), max(y, 0)), np.int64)
    rho = C.c_double()
    _check(load_library().dbsp_ring_work(_ptr(mask), H, nQ, nK, y, _ptr(gq), _ptr(gk), _ptr(work), C.byref(rho)))
    return work.tolist(), rho.value


def fit_cost_model(blocks, items, time):
    """Least-squares (a, c, t0, rms residual) of time = a*blocks + c*items + t0 (see dbsp.h: dbsp_fit_cost_model)."""
    b = np.ascontiguousarray(blocks, dtype=np.int64)
    i = np.ascontiguousarray(items, dtype=np.int64)
    t = np.ascontiguousarray(time, dtype=np.float64)
    if not (b.shape == i.shape == t.shape and b.ndim == 1):
        raise ValueError("blocks, items and time must be 1-D arrays of one length")
    a, c, t0, rms = C.c_double(), C.c_double(), C.c_double(), C.c_double()
    _check(load_library().dbsp_fit_cost_model(_ptr(b), _ptr(i), _ptr(t), b.shape[0], C.byref(a), C.byref(c), C.byref(t0), C.byref(rms)))
    return a.value, c.value, t0.value, rms.value


def mfma_probe(stream=None):
    """(sustained dense bf16 MFMA TFLOP/s, shader clock in GHz) measured on the current device (see dbsp.h: dbsp_mfma_probe)."""
    t, g = C.c_double(), C.c_double()
    _check(load_library().dbsp_mfma_probe(C.byref(t), C.byref(g), _stream_ptr(stream)))
    return t.value, g.value
