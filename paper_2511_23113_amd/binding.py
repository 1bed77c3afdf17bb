"""ctypes binding of libdbsp's C ABI (include/dbsp.h): argument marshalling only.

Every step of the hot path runs inside the library; nothing here computes.  The library is
loaded from this package's directory; if it has not been built yet it is built once with
hipcc, and any failure to build or load raises -- there is no CPU fallback.
"""

from __future__ import annotations

import copy
import ctypes as C
import os

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


class KVCache:
    """A key/value cache of the caller's tensors (see dbsp.h: dbsp_cache), for cache_attn_fwd and cache_evict.

    k, v: [B, Hk, capacity, d], bf16 or fp16 on one GPU, d in (64, 128) dense, other strides multiples of 8 elements; the first
    lens[b] (int32 [B] there) slots of sequence b are used.  prefix_k, prefix_v: [Hk, P, d], shared by all sequences.  Either
    pair may be missing.  weights: f32 [B, Hk, capacity], positions: int32 [B, Hk, capacity], both contiguous.  The object keeps the
    tensors, which the caller goes on writing; it copies nothing, and other tensors make another object."""

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
        self._desc, self._at, self._bytes, self._index = desc, C.byref(desc), {}, self.device.index

    def _for(self, B):
        """The same prefix for B sequences."""
        other = copy.copy(self)
        other._desc = CacheDesc.from_buffer_copy(self._desc)
        other._desc.B = other.B = B
        other._at, other._bytes = C.byref(other._desc), {}
        return other

    def _on(self, stream):
        """The raw stream, and whether tensors made on torch's current one are used on another."""
        torch = _torch
        if self._index != torch._C._cuda_getDevice():
            raise ValueError("the cache lives on another device than the current one")
        now = torch._C._cuda_getCurrentRawStream(self._index)
        if stream is None:
            return now, False
        if isinstance(stream, int):
            return stream, stream != now
        if getattr(stream, "device", self.device) != self.device:
            raise ValueError("the stream is of another device than the cache")
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


def cache_attn_fwd(cache: KVCache, q, q_lens=None, causal: bool = True, decay=None, o=None, lse=None, softmax_scale: float = 0.0,
                   stream=None, want_lse: bool = True, workspace=None):
    """Attention of each sequence's newest tokens, q [B, H, Nq, d], over the cache's shared prefix and its own keys (see dbsp.h:
    dbsp_cache_attn_fwd; the new tokens' keys are written before).  q_lens: int32 [B] on the GPU, if not all Nq tokens are there;
    the others' rows of o and lse are left as they were, so pass o and lse then.  decay: None, or the factor of what the cache's
    weights hold, to which this call's attention is added.  Enqueues on `stream` (default: torch's current stream) and
    returns (o, lse)."""
    torch = _torch
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
    raw, elsewhere = cache._on(stream)
    if keep_from is not None and (keep_from.shape != (cache.B,) or keep_from.dtype != torch.int32 or keep_from.device != cache.device or not keep_from.is_contiguous()):
        raise ValueError("keep_from must be a contiguous int32 tensor of [B] on the cache's GPU")
    workspace, at, size = cache._workspace(workspace, (budget,), _lib.dbsp_cache_evict_workspace, raw, elsewhere)
    rc = _lib.dbsp_cache_evict(cache._at, budget, sinks, None if keep_from is None else keep_from.data_ptr(), at, size, raw)
    if rc:
        _check(rc)


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
