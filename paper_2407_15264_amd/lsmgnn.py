"""Python binding of the MI355X feature-gather cache (C ABI in include/lsmgnn.h).

Argument marshalling only: every step of a gather runs in the gfx950 kernels of
liblsmgnn.so.  PyTorch supplies device memory (tensors) and the stream.  There
is no CPU fallback: if the library is missing this module raises.
"""
from __future__ import annotations

import atexit
import ctypes
import os
import weakref

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "liblsmgnn.so")

OK, E_INVAL, E_RANGE, E_WINDOW, E_NOMEM, E_DEVICE, E_STATE = range(7)
STATUS_NAMES = {0: "OK", 1: "E_INVAL", 2: "E_RANGE", 3: "E_WINDOW", 4: "E_NOMEM", 5: "E_DEVICE", 6: "E_STATE"}
HIT, VICTIM_HIT, MISS = 0, 1, 2
EMPTY = 0xFFFFFFFF
COUNT_FIELDS = ("batch", "requests", "unique", "hits", "victim_hits", "misses", "evictions", "enqueued",
                "dropped", "request_hits", "request_victim_hits", "victim_rows_ring", "victim_rows_staged",
                "victim_rows_cache", "victim_rows_prefetched")


class LsmgnnError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        self.status = STATUS_NAMES.get(code, str(code))
        msg = lib().lsmgnn_strerror(code).decode() if _lib is not None else self.status
        super().__init__(f"{where}: {self.status} ({msg})")


class Config(ctypes.Structure):
    _fields_ = [("num_nodes", ctypes.c_uint64), ("row_bytes", ctypes.c_uint64), ("num_sets", ctypes.c_uint64),
                ("victim_rows", ctypes.c_uint64), ("max_batch", ctypes.c_uint64), ("lookahead", ctypes.c_uint32),
                ("near_threshold", ctypes.c_uint32), ("device", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("host_threads", ctypes.c_uint32), ("policy", ctypes.c_uint32), ("victim_mode", ctypes.c_uint32),
                ("refresh_period", ctypes.c_uint32), ("host_store", ctypes.c_void_p),
                ("static_score", ctypes.c_void_p)]


FLAG_PAGEABLE_STORE = 1
# lsmgnn_config.policy values: the method's hybrid order and the evaluation's
# alternatives (static score only, next announced use only, round-robin)
POLICY = {"hybrid": 0, "static": 1, "dynamic": 2, "round_robin": 3}
# lsmgnn_config.victim_mode values: one FIFO ring, or per-reuse-iteration
# queues prefetched into HBM before their iteration
VICTIM_MODE = {"fifo": 0, "queues": 1}


class Counts(ctypes.Structure):
    _fields_ = [(f, ctypes.c_uint64) for f in COUNT_FIELDS]


class Profile(ctypes.Structure):
    _fields_ = [("hbm_copy_ms", ctypes.c_double), ("hbm_copy_launches", ctypes.c_uint64),
                ("hbm_copy_rows", ctypes.c_uint64),
                ("host_fetch_ms", ctypes.c_double), ("host_fetch_launches", ctypes.c_uint64),
                ("host_fetch_rows", ctypes.c_uint64),
                ("enqueue_ms", ctypes.c_double), ("enqueue_launches", ctypes.c_uint64),
                ("enqueue_rows", ctypes.c_uint64),
                ("fill_ms", ctypes.c_double), ("fill_launches", ctypes.c_uint64), ("fill_rows", ctypes.c_uint64),
                ("host_copy_ms", ctypes.c_double), ("host_copy_rows", ctypes.c_uint64),
                ("prefetch_ms", ctypes.c_double), ("prefetch_launches", ctypes.c_uint64),
                ("prefetch_rows", ctypes.c_uint64),
                ("gather_ms", ctypes.c_double), ("gathers", ctypes.c_uint64)]


_lib = None

# Library objects still open, closed at interpreter exit before module
# teardown begins: caches first (their host threads read the stores and their
# streams may still move rows), then samplers, then pinned buffers.  A
# finalizer that ran during teardown would find the module's globals gone.
_LIVE = {"cache": weakref.WeakSet(), "sampler": weakref.WeakSet(), "pinned": weakref.WeakSet()}


def _close_all():
    for kind in ("cache", "sampler", "pinned"):
        for obj in list(_LIVE[kind]):
            obj.close()


atexit.register(_close_all)


def lib():
    """Load liblsmgnn.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(hipcc --offload-arch=gfx950); there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, u64, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int
        L.lsmgnn_cache_create.restype = i32
        L.lsmgnn_cache_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(vp)]
        L.lsmgnn_cache_destroy.restype = None
        L.lsmgnn_cache_destroy.argtypes = [vp]
        L.lsmgnn_advance.restype = i32
        L.lsmgnn_advance.argtypes = [vp, vp, u64, vp]
        L.lsmgnn_gather.restype = i32
        L.lsmgnn_gather.argtypes = [vp, vp, u64, vp, vp, vp, vp, ctypes.POINTER(u64), vp]
        L.lsmgnn_gather_async.restype = i32
        L.lsmgnn_gather_async.argtypes = [vp, vp, u64, vp, u64, vp, vp, vp, vp, ctypes.POINTER(u64),
                                          ctypes.POINTER(u64), vp]
        L.lsmgnn_gather_wait.restype = i32
        L.lsmgnn_gather_wait.argtypes = [vp, u64, vp]
        L.lsmgnn_sync.restype = i32
        L.lsmgnn_sync.argtypes = [vp]
        L.lsmgnn_stats.restype = i32
        L.lsmgnn_stats.argtypes = [vp, ctypes.POINTER(Counts), ctypes.POINTER(Counts)]
        L.lsmgnn_export_state.restype = i32
        L.lsmgnn_export_state.argtypes = [vp, vp, vp, ctypes.POINTER(u64), ctypes.POINTER(u64)]
        L.lsmgnn_set_profiling.restype = i32
        L.lsmgnn_set_profiling.argtypes = [vp, i32]
        L.lsmgnn_get_profile.restype = i32
        L.lsmgnn_get_profile.argtypes = [vp, ctypes.POINTER(Profile)]
        L.lsmgnn_host_alloc.restype = i32
        L.lsmgnn_host_alloc.argtypes = [u64, ctypes.POINTER(vp)]
        L.lsmgnn_host_free.restype = None
        L.lsmgnn_host_free.argtypes = [vp]
        L.lsmgnn_set_of.restype = u64
        L.lsmgnn_set_of.argtypes = [u64, u64]
        L.lsmgnn_copy_bytes.restype = i32
        L.lsmgnn_copy_bytes.argtypes = [vp, vp, u64, vp]
        L.lsmgnn_pagerank_scores.restype = i32
        L.lsmgnn_pagerank_scores.argtypes = [vp, vp, u64, ctypes.c_double, ctypes.c_uint32, vp, vp, i32, vp]
        L.lsmgnn_expand.restype = i32
        L.lsmgnn_expand.argtypes = [vp, vp, u64, u64, vp, vp]
        L.lsmgnn_sampler_create.restype = i32
        L.lsmgnn_sampler_create.argtypes = [vp, vp, u64, vp, ctypes.c_uint32, u64, i32, ctypes.POINTER(vp)]
        L.lsmgnn_sampler_destroy.restype = None
        L.lsmgnn_sampler_destroy.argtypes = [vp]
        L.lsmgnn_sample.restype = i32
        L.lsmgnn_sample.argtypes = [vp, vp, u64, u64, vp, u64, ctypes.POINTER(u64), vp]
        L.lsmgnn_sample_async.restype = i32
        L.lsmgnn_sample_async.argtypes = [vp, vp, u64, u64, vp, u64, vp, vp]
        L.lsmgnn_split_work_bytes.restype = u64
        L.lsmgnn_split_work_bytes.argtypes = [u64, ctypes.c_uint32]
        L.lsmgnn_split_by_type_async.restype = i32
        L.lsmgnn_split_by_type_async.argtypes = [vp, u64, u64, vp, vp, ctypes.c_uint32, ctypes.POINTER(vp), u64,
                                                 vp, u64, vp, vp]
        L.lsmgnn_split_by_type_noalloc_async.restype = i32
        L.lsmgnn_split_by_type_noalloc_async.argtypes = [vp, u64, u64, vp, vp, ctypes.c_uint32, ctypes.POINTER(vp),
                                                         u64, vp, vp]
        u32, i64, f32 = ctypes.c_uint32, ctypes.c_int64, ctypes.c_float
        for name, res, args in (
                ("embed_rows", i32, [vp, u64, u64, u64, u32, vp, u64, i64, f32, vp, u64, u32, vp, vp]),
                ("embed_grad_work_bytes", u64, [u64, u64, u64]),
                ("table_grad_work_bytes", u64, [u64, u64, u64]),
                ("embed_grad", i32, [vp, u64, u64, u32, vp, u64, u64, i64, f32, vp, u64, u32, vp, u64, vp, vp]),
                ("embed_grad_rows", i32, [vp, u64, u64, u32, vp, u64, u64, i64, f32, vp, vp, u64, u32, vp, u64, vp,
                                          vp]),
                ("route_max_rows", u64, [u64, u32, u32, u32]),
                ("route_work_bytes", u64, [u64, u32, u32]),
                ("route_plan", i32, [vp, u64, u32, u32, u32, vp, vp, vp, vp, u64, vp, vp]),
                ("route_rows", i32, [vp, u64, u64, u64, u32, vp, vp, u32, u64, vp, u64, vp]),
                ("route_combine", i32, [vp, u64, u64, u64, u32, vp, vp, u64, u32, vp, u64, vp]),
                ("route_combine_grad", i32, [vp, u64, u64, u64, u32, vp, u64, vp, vp, vp, u32, u64, vp, u64, vp, vp]),
                ("pack_blocks", u64, [u64]),
                ("pack8", i32, [vp, u64, u64, u64, u32, vp, vp, vp]),
                ("unpack8", i32, [vp, vp, u64, u64, vp, u64, u32, vp]),
                ("act8", i32, [vp, u64, u64, u64, u32, u32, u32, vp, u64, vp, vp, vp]),
                ("act8_grad", i32, [vp, u64, u64, u64, u32, vp, vp, u32, u32, vp, u64, vp]),
                ("weight_grad8_work_bytes", u64, [u64, u64, u64, u32]),
                ("weight_grad8", i32, [vp, vp, u64, u64, vp, u64, u64, u32, vp, u32, vp, u32, vp, u64, vp])):
            fn = getattr(L, "lsmgnn_" + name)
            fn.restype, fn.argtypes = res, args
        L.lsmgnn_strerror.restype = ctypes.c_char_p
        L.lsmgnn_strerror.argtypes = [i32]
        _lib = L
    return _lib


def _check(rc: int, where: str):
    if rc != OK:
        raise LsmgnnError(rc, where)


def set_of(x: int, num_sets: int) -> int:
    return int(lib().lsmgnn_set_of(int(x), int(num_sets)))


def copy_bytes(dst_ptr: int, src_ptr: int, nbytes: int, stream=None, device=0):
    """Calibration copy (device or pinned host pointers), synchronous."""
    _check(lib().lsmgnn_copy_bytes(ctypes.c_void_p(dst_ptr), ctypes.c_void_p(src_ptr), int(nbytes),
                                   _stream_handle(stream, device)), "lsmgnn_copy_bytes")


def expand(rows, inverse, row_bytes, out=None, stream=None, device=0):
    """Rows in request order (lsmgnn_expand): out[i] = rows[inverse[i]].  rows:
    a gather's unique-row output (uint8 device tensor), inverse: its int64
    inverse index (n entries).  Returns `out` (uint8, n * row_bytes), allocated
    when not given."""
    import torch
    n = inverse.numel()
    if out is None:
        out = torch.empty(max(n, 1) * row_bytes, dtype=torch.uint8, device=inverse.device)
    _check(lib().lsmgnn_expand(ctypes.c_void_p(rows.data_ptr()), ctypes.c_void_p(inverse.data_ptr()), n,
                               int(row_bytes), ctypes.c_void_p(out.data_ptr()), _stream_handle(stream, device)),
           "lsmgnn_expand")
    return out[: n * row_bytes]


def pagerank_scores(offsets, adj, damping=0.85, iterations=20, rank=False, device=0, stream=None):
    """Reverse-PageRank static scores (lsmgnn_pagerank_scores) of a CSR graph
    given as device tensors (offsets int64 [N+1], adj int32/uint32 [E]).
    Returns a device uint32-valued int32 tensor of scores (viewed as uint32 by
    callers through .cpu().numpy().view(np.uint32)), and the float64 ranks
    when rank=True."""
    import torch
    dev = torch.device("cuda", device)
    n = offsets.numel() - 1
    scores = torch.empty(max(n, 1), dtype=torch.int32, device=dev)
    rk = torch.empty(max(n, 1), dtype=torch.float64, device=dev) if rank else None
    _check(lib().lsmgnn_pagerank_scores(ctypes.c_void_p(offsets.data_ptr()),
                                        ctypes.c_void_p(adj.data_ptr()) if adj.numel() else None, n,
                                        float(damping), int(iterations), ctypes.c_void_p(scores.data_ptr()),
                                        ctypes.c_void_p(rk.data_ptr()) if rank else None, int(device),
                                        _stream_handle(stream, device)), "lsmgnn_pagerank_scores")
    return (scores[:n], rk[:n]) if rank else scores[:n]


class GpuSampler:
    """GraphSAGE request lists sampled on the GPU (lsmgnn_sampler_create /
    lsmgnn_sample) from a CSR graph in device memory (offsets int64 [N+1],
    adj int32/uint32 [E]); the tensors must outlive the sampler."""

    def __init__(self, offsets, adj, fanout, seed=0, device=0):
        import torch
        self.device = torch.device("cuda", device)
        off_p = _dev_ptr(offsets, torch.int64, "offsets")
        adj_p = _dev_ptr(adj, (torch.int32, torch.uint32), "adj") if adj.numel() else None
        self._graph = (offsets, adj)  # keeps the borrowed graph alive
        self.num_nodes = offsets.numel() - 1
        fan = (ctypes.c_uint32 * len(fanout))(*[int(f) for f in fanout])
        self.hops = len(fanout)
        h = ctypes.c_void_p()
        _check(lib().lsmgnn_sampler_create(off_p, adj_p, self.num_nodes, fan, self.hops, int(seed), int(device),
                                           ctypes.byref(h)), "lsmgnn_sampler_create")
        self._destroy = lib().lsmgnn_sampler_destroy  # kept: module globals may be gone when the finalizer runs
        self._h = h
        _LIVE["sampler"].add(self)

    def close(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    __del__ = close

    def sample(self, seeds, batch, out, stream=None):
        """Request list of minibatch `batch` from its seeds (int64 device
        tensor) into `out` (int64 device tensor); returns out[:length]."""
        import torch
        sp = _dev_ptr(seeds, torch.int64, "seeds") if seeds.numel() else None
        op = _dev_ptr(out, torch.int64, "out")
        n = ctypes.c_uint64(0)
        _check(lib().lsmgnn_sample(self._h, sp, seeds.numel(), int(batch), op, out.numel(), ctypes.byref(n),
                                   _stream_handle(stream, self.device.index)), "lsmgnn_sample")
        return out[: n.value]

    def sample_async(self, seeds, batch, out, result_ptr, stream=None):
        """Queue the sampling of minibatch `batch` into `out`; once `stream`
        has run it, the two uint64 at result_ptr (pinned host memory) hold
        the list's length and its status code."""
        import torch
        sp = _dev_ptr(seeds, torch.int64, "seeds") if seeds.numel() else None
        op = _dev_ptr(out, torch.int64, "out")
        _check(lib().lsmgnn_sample_async(self._h, sp, seeds.numel(), int(batch), op, out.numel(),
                                         ctypes.c_void_p(result_ptr), _stream_handle(stream, self.device.index)),
               "lsmgnn_sample_async")


def split_work_bytes(n, num_types):
    """Device work memory split_by_type_async needs for n requests."""
    return int(lib().lsmgnn_split_work_bytes(int(n), int(num_types)))


def split_by_type_async(ids, node_type, local, outs, work, result_ptr, stream=None, device=0):
    """Queue the split of a global request list (int64 device tensor) into one
    list of within-type indices per node type (lsmgnn_split_by_type_async):
    node_type (uint8 device tensor), local (int32/uint32 device tensor), outs
    (int64 device tensors of equal length, one per type), work (a device
    tensor of at least split_work_bytes bytes); result_ptr: pinned host
    memory for the len(outs) lengths and the status."""
    import torch
    T = len(outs)
    if T == 0:
        raise ValueError("outs must hold one tensor per node type")
    ids_p = _dev_ptr(ids, torch.int64, "ids") if ids.numel() else None
    type_p = _dev_ptr(node_type, torch.uint8, "node_type")
    local_p = _dev_ptr(local, (torch.int32, torch.uint32), "local")
    if local.numel() != node_type.numel():
        raise ValueError("local and node_type must have one entry per node")
    ptrs = (ctypes.c_void_p * T)(*[_dev_ptr(o, torch.int64, f"outs[{t}]").value for t, o in enumerate(outs)])
    cap = min(o.numel() for o in outs)  # every list may be written up to the capacity
    work_p = _dev_ptr(work, work.dtype, "work")
    _check(lib().lsmgnn_split_by_type_async(ids_p, ids.numel(), node_type.numel(), type_p, local_p, T, ptrs, cap,
                                            work_p, work.numel() * work.element_size(),
                                            ctypes.c_void_p(result_ptr), _stream_handle(stream, device)),
           "lsmgnn_split_by_type_async")


def split_by_type_noalloc_async(ids, node_type, local, outs, result_ptr, stream=None, device=0):
    """split_by_type_async without the work tensor
    (lsmgnn_split_by_type_noalloc_async): the library's own device array is
    the work memory, so the call allocates nothing; calls that may overlap on
    one device must be ordered by the caller."""
    import torch
    T = len(outs)
    if T == 0:
        raise ValueError("outs must hold one tensor per node type")
    ids_p = _dev_ptr(ids, torch.int64, "ids") if ids.numel() else None
    type_p = _dev_ptr(node_type, torch.uint8, "node_type")
    local_p = _dev_ptr(local, (torch.int32, torch.uint32), "local")
    if local.numel() != node_type.numel():
        raise ValueError("local and node_type must have one entry per node")
    ptrs = (ctypes.c_void_p * T)(*[_dev_ptr(o, torch.int64, f"outs[{t}]").value for t, o in enumerate(outs)])
    cap = min(o.numel() for o in outs)
    _check(lib().lsmgnn_split_by_type_noalloc_async(ids_p, ids.numel(), node_type.numel(), type_p, local_p, T, ptrs,
                                                    cap, ctypes.c_void_p(result_ptr), _stream_handle(stream, device)),
           "lsmgnn_split_by_type_noalloc_async")


class PinnedBuffer:
    """Exact-size pinned, device-mapped host memory (lsmgnn_host_alloc)."""

    def __init__(self, nbytes: int):
        p = ctypes.c_void_p()
        _check(lib().lsmgnn_host_alloc(int(nbytes), ctypes.byref(p)), "lsmgnn_host_alloc")
        self.ptr = p.value
        self.nbytes = int(nbytes)
        self._free = lib().lsmgnn_host_free  # kept: module globals may be gone when the finalizer runs
        _LIVE["pinned"].add(self)

    def numpy(self, dtype=np.uint8, shape=None) -> np.ndarray:
        raw = (ctypes.c_uint8 * self.nbytes).from_address(self.ptr)
        a = np.frombuffer(raw, dtype=np.uint8).view(dtype)
        return a if shape is None else a.reshape(shape)

    def close(self):
        if getattr(self, "ptr", None):
            self._free(self.ptr)
            self.ptr = None

    __del__ = close


def _stream_handle(stream, device):
    import torch
    s = torch.cuda.current_stream(device) if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dev_ptr(t, dtype, name):
    """Device address of a contiguous tensor of `dtype` (or one of a tuple of
    dtypes); raises TypeError for anything else."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    ok = t.dtype in dtype if isinstance(dtype, tuple) else t.dtype == dtype
    if not ok or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor")
    return ctypes.c_void_p(t.data_ptr())


class GatherResult:
    """Outputs of one gather as views of the caller's buffers (built on first
    access, so the hot loop pays nothing for them):
    out (n_unique, row_bytes) uint8, unique (n_unique,) int64, inverse (n,)
    int64 or None, outcome (n_unique,) uint8 or None."""

    __slots__ = ("n_unique", "n", "row_bytes", "_out", "_unique", "_inverse", "_outcome")

    def __init__(self, n_unique, n, row_bytes, out, unique, inverse, outcome):
        self.n_unique, self.n, self.row_bytes = n_unique, n, row_bytes
        self._out, self._unique, self._inverse, self._outcome = out, unique, inverse, outcome

    @property
    def out(self):
        import torch
        U = self.n_unique
        return self._out.view(torch.uint8).reshape(-1)[: U * self.row_bytes].view(U, self.row_bytes)

    @property
    def unique(self):
        return self._unique[: self.n_unique]

    @property
    def inverse(self):
        return None if self._inverse is None else self._inverse[: self.n]

    @property
    def outcome(self):
        return None if self._outcome is None else self._outcome[: self.n_unique]


class FeatureCache:
    """GPU feature-gather cache on one device.

    host_store: num_nodes * row_bytes bytes of host memory that must outlive
    the cache: pinned (a PinnedBuffer, its ptr, or a pinned torch tensor), or
    with pageable=True ordinary memory (a numpy array or an address), whose
    rows the library's host threads (host_threads, 0 = 8) copy for the GPU.
    static_score: num_nodes unsigned scores.
    policy: a name in POLICY (or its number); victim_mode: a name in
    VICTIM_MODE (or its number); refresh_period: the update period of the
    dynamic information (1 = exact at every gather)."""

    def __init__(self, num_nodes, row_bytes, host_store, static_score, num_sets, victim_rows, lookahead,
                 max_batch, near_threshold=0, device=0, pageable=False, host_threads=0, policy="hybrid",
                 victim_mode="fifo", refresh_period=1):
        import torch
        self.device = torch.device("cuda", device)
        self.num_nodes, self.row_bytes = int(num_nodes), int(row_bytes)
        self.num_sets, self.victim_rows = int(num_sets), int(victim_rows)
        self.lookahead, self.max_batch = int(lookahead), int(max_batch)
        if isinstance(host_store, PinnedBuffer):
            host_store = host_store.ptr
        elif isinstance(host_store, torch.Tensor):
            host_store = host_store.data_ptr()
        elif isinstance(host_store, np.ndarray):
            if not host_store.flags.c_contiguous or host_store.nbytes < self.num_nodes * self.row_bytes:
                raise ValueError("host_store array must be C-contiguous and hold num_nodes * row_bytes bytes")
            self._store_ref = host_store
            host_store = host_store.ctypes.data
        stat = np.ascontiguousarray(np.asarray(static_score), dtype=np.uint32)
        cfg = Config(self.num_nodes, self.row_bytes, self.num_sets, self.victim_rows, self.max_batch,
                     self.lookahead, int(near_threshold), int(device), FLAG_PAGEABLE_STORE if pageable else 0,
                     int(host_threads), int(POLICY.get(policy, policy)),
                     int(VICTIM_MODE.get(victim_mode, victim_mode)), int(refresh_period),
                     ctypes.c_void_p(int(host_store)),
                     ctypes.c_void_p(stat.ctypes.data))
        h = ctypes.c_void_p()
        _check(lib().lsmgnn_cache_create(ctypes.byref(cfg), ctypes.byref(h)), "lsmgnn_cache_create")
        self._destroy = lib().lsmgnn_cache_destroy  # kept: module globals may be gone when the finalizer runs
        self._h = h
        self._scratch = {}
        _LIVE["cache"].add(self)

    def close(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    __del__ = close

    def _buf(self, name, n, dtype):
        import torch
        b = self._scratch.get(name)
        if b is None or b.numel() < n:
            b = torch.empty(max(n, 1), dtype=dtype, device=self.device)
            self._scratch[name] = b
        return b

    def advance(self, ids, stream=None):
        import torch
        n = ids.numel()
        p = _dev_ptr(ids, torch.int64, "ids") if n else None
        _check(lib().lsmgnn_advance(self._h, p, n, _stream_handle(stream, self.device)), "lsmgnn_advance")

    def _gather_args(self, ids, out, unique, inverse, outcome):
        import torch
        n = ids.numel()
        if out is None:
            out = self._buf("out", n * self.row_bytes, torch.uint8)
        if unique is None:
            unique = self._buf("unique", n, torch.int64)

        def pick(arg, name, dtype):
            if isinstance(arg, torch.Tensor):
                if arg.numel() < n:
                    raise ValueError(f"{name} buffer too small")
                return arg
            return self._buf(name, n, dtype) if arg else None

        inv_t = pick(inverse, "inverse", torch.int64)
        oc_t = pick(outcome, "outcome", torch.uint8)
        if out.numel() * out.element_size() < n * self.row_bytes or unique.numel() < n:
            raise ValueError("out/unique buffers too small")
        args = (self._h, _dev_ptr(ids, torch.int64, "ids") if n else None, n,
                ctypes.c_void_p(out.data_ptr()), _dev_ptr(unique, torch.int64, "unique"),
                _dev_ptr(inv_t, torch.int64, "inverse") if inv_t is not None else None,
                _dev_ptr(oc_t, torch.uint8, "outcome") if oc_t is not None else None)
        return n, out, unique, inv_t, oc_t, args

    def _result(self, U, n, out, unique, inv_t, oc_t):
        return GatherResult(U, n, self.row_bytes, out, unique, inv_t, oc_t)

    def gather(self, ids, out=None, unique=None, inverse=True, outcome=False, stream=None) -> GatherResult:
        """Gather one minibatch (returns when everything is complete).  `out`
        (uint8, >= n*row_bytes bytes) and `unique` (int64, >= n) may be passed
        to reuse caller buffers; `inverse`/`outcome` may be True (allocate), a
        tensor, or False/None."""
        n, out, unique, inv_t, oc_t, args = self._gather_args(ids, out, unique, inverse, outcome)
        nu = ctypes.c_uint64()
        _check(lib().lsmgnn_gather(*args, ctypes.byref(nu), _stream_handle(stream, self.device)), "lsmgnn_gather")
        return self._result(nu.value, n, out, unique, inv_t, oc_t)

    def gather_async(self, ids, out, unique, inverse=None, outcome=None, stream=None, announce=None):
        """Pipelined gather: returns (ticket, GatherResult) once the unique
        count is known.  `announce` (int64 device tensor, or None) is the next
        minibatch to announce after this gather, as advance() would.  The
        buffers must be caller-owned tensors (not reused until wait(ticket) and
        a synchronisation of the stream)."""
        import torch
        n, out, unique, inv_t, oc_t, args = self._gather_args(ids, out, unique, inverse, outcome)
        if announce is None:
            ann = (None, 0)
        else:
            an = announce.numel()
            # any non-NULL pointer announces, even an empty list (then it is
            # not read): the unique buffer's address serves
            ann = (_dev_ptr(announce, torch.int64, "announce") if an else args[4], an)
        nu, tk = ctypes.c_uint64(), ctypes.c_uint64()
        _check(lib().lsmgnn_gather_async(*args[:3], *ann, *args[3:], ctypes.byref(nu), ctypes.byref(tk),
                                         _stream_handle(stream, self.device)), "lsmgnn_gather_async")
        return tk.value, self._result(nu.value, n, out, unique, inv_t, oc_t)

    def wait(self, ticket, stream=None):
        """Make `stream` wait (on the device) for gather `ticket`."""
        _check(lib().lsmgnn_gather_wait(self._h, int(ticket), _stream_handle(stream, self.device)),
               "lsmgnn_gather_wait")

    def sync(self):
        _check(lib().lsmgnn_sync(self._h), "lsmgnn_sync")

    def stats(self):
        last, total = Counts(), Counts()
        _check(lib().lsmgnn_stats(self._h, ctypes.byref(last), ctypes.byref(total)), "lsmgnn_stats")
        return ({f: getattr(last, f) for f in COUNT_FIELDS}, {f: getattr(total, f) for f in COUNT_FIELDS})

    def export_state(self):
        tags = np.empty(self.num_sets * 8, np.uint32)
        ring = np.empty(max(self.victim_rows, 1), np.uint32)
        tail, t = ctypes.c_uint64(), ctypes.c_uint64()
        _check(lib().lsmgnn_export_state(self._h, tags.ctypes.data, ring.ctypes.data, ctypes.byref(tail),
                                         ctypes.byref(t)), "lsmgnn_export_state")
        return dict(tags=tags.reshape(self.num_sets, 8), ring_tags=ring[: self.victim_rows],
                    ring_tail=tail.value, t=t.value)

    def set_profiling(self, on: bool):
        _check(lib().lsmgnn_set_profiling(self._h, 1 if on else 0), "lsmgnn_set_profiling")

    def profile(self) -> dict:
        p = Profile()
        _check(lib().lsmgnn_get_profile(self._h, ctypes.byref(p)), "lsmgnn_get_profile")
        return {f: getattr(p, f) for f, _ in Profile._fields_}


# ------------------------------------------------------------- trained rows
# lsmgnn.h's element types and activations
ELEMENT_TYPES = {"float32": 0, "float16": 1, "bfloat16": 2}
ACTIVATIONS = {"silu": 0, "gelu": 1}
NO_PAD = -(1 << 63)
PACK_BLOCK = 32

_TYPE_CODES = {}  # torch dtype -> element type


def _type_code(dtype, name):
    if not _TYPE_CODES:
        import torch
        _TYPE_CODES.update({getattr(torch, n): c for n, c in ELEMENT_TYPES.items()})
    code = _TYPE_CODES.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, not {dtype}")
    return code


def _no_graph(t, name):
    """Refuse a tensor whose gradient torch would expect to hear of: the calls below
    record nothing, and their results would silently end the graph."""
    import torch
    if torch.is_grad_enabled():
        raise RuntimeError(f"{name} requires a gradient, which this call does not record: call it under "
                           "torch.no_grad() or from a torch.autograd.Function, with the gradient's own call")


def _matrix(t, name, dim=None, rows=None, like=None):
    """(address, rows, dim, ld, element type) of a 2-D device tensor whose rows
    are contiguous; with `like`, of the same device."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.requires_grad:
        _no_graph(t, name)
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, not {t.dim()}")
    n, d = t.shape
    row, column = t.stride()
    ld = row if n > 1 else max(d, 1)
    if d > 1 and column != 1 or ld < d:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    if dim is not None and d != dim or rows is not None and n != rows:
        raise ValueError(f"{name} must be {rows if rows is not None else n} rows of {dim if dim is not None else d}, "
                         f"not {n} of {d}")
    if like is not None and t.device != like:
        raise ValueError(f"{name} is on {t.device}, not on {like}")
    return t.data_ptr(), n, d, ld, _type_code(t.dtype, name)


def _vector(t, dtype, numel, name, device, floats=False):
    """Address of a contiguous device tensor of `numel` elements of `dtype`, a
    floating-point one or not."""
    _dev_ptr(t, dtype, name)
    if floats and t.requires_grad:
        _no_graph(t, name)
    if t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements, not {t.numel()}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return t.data_ptr()


_raw_stream = _raw_device = None


def _run(name, device, stream, *args):
    """Call the library's `name` on `stream` (None: the current one of `device`, the
    tensors' device) with that device current: the handle of a default stream, 0, is
    the current device's.  Looked up without making a Stream object: 0.1 us against
    2."""
    global _raw_stream, _raw_device
    if _raw_stream is None:
        import torch
        _raw_stream, _raw_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    index = device.index
    if stream is None:
        handle = _raw_stream(index)
    else:
        if stream.device != device:
            raise ValueError(f"stream is of {stream.device}, not of {device}")
        handle = stream.cuda_stream
    fn = getattr(lib(), name)
    if _raw_device() == index:
        rc = fn(*args, handle)
    else:
        import torch
        with torch.cuda.device(device):
            rc = fn(*args, handle)
    if rc:
        _check(rc, name)


def _empty(shape, dtype, device, stream):
    """Device memory for work on `stream` (None: the current one), from that
    stream's pool, so that its reuse after a free is ordered behind the work."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _output(t, name, rows, dim, dtype, device, stream):
    """(tensor, address, ld, element type) of an output: the caller's, checked, or
    one allocated here."""
    if t is None:
        t = _empty((rows, dim), dtype, device, stream)
        return t, t.data_ptr(), dim, _type_code(dtype, name)
    p, _, _, ld, code = _matrix(t, name, dim, rows, device)
    return t, p, ld, code


def _work(nbytes, work, device, stream):
    if work is None:
        if nbytes == 0:
            return None, None, 0
        import torch
        work = _empty(nbytes, torch.uint8, device, stream)
    _dev_ptr(work, work.dtype, "work")
    if work.device != device:
        raise ValueError(f"work is on {work.device}, not on {device}")
    return work, work.data_ptr(), work.numel() * work.element_size()


def embed_rows(table, ids, scale=1.0, pad=None, dtype=None, out=None, status_ptr=None, stream=None):
    """Rows of a trained table (lsmgnn_embed_rows): out[i] = scale *
    table[ids[i]], zeros where ids[i] == pad.  table: (num_rows, dim) device
    tensor, ids: int64 device tensor (n entries).  Returns out (n, dim), of
    `dtype` (default the table's) where it is allocated here; on a stream of the
    caller's it comes from that stream's pool.  status_ptr: address of a uint64
    that receives E_RANGE for an ID out of range."""
    import torch
    device = table.device
    tp, num_rows, dim, tld, tt = _matrix(table, "table")
    n = ids.numel()
    ip = _vector(ids, torch.int64, n, "ids", device)
    out, op, old, ot = _output(out, "out", n, dim, dtype or table.dtype, device, stream)
    _run("lsmgnn_embed_rows", device, stream, tp, num_rows, dim, tld, tt, ip, n, NO_PAD if pad is None else pad,
         scale, op, old, ot, status_ptr)
    return out


def embed_grad_work_bytes(n, num_rows, dim):
    """Device work memory the gradient of a lookup of n IDs needs, whole or by rows."""
    return int(lib().lsmgnn_embed_grad_work_bytes(int(n), int(num_rows), int(dim)))


def table_grad_work_bytes(n, num_rows, dim):
    """Device work memory the whole gradient needs: none where one launch does it."""
    return int(lib().lsmgnn_table_grad_work_bytes(int(n), int(num_rows), int(dim)))


def embed_grad(dy, ids, num_rows, scale=1.0, pad=None, dtype=None, grad=None, work=None, status_ptr=None,
               stream=None):
    """The whole gradient of embed_rows' table (lsmgnn_embed_grad), (num_rows,
    dim) of `dtype` (default dy's) or into `grad`.  dy: (n, dim) device tensor,
    ids: the lookup's."""
    import torch
    device = dy.device
    dp, n, dim, dld, dt = _matrix(dy, "dy")
    ip = _vector(ids, torch.int64, n, "ids", device)
    grad, gp, gld, gt = _output(grad, "grad", num_rows, dim, dtype or dy.dtype, device, stream)
    work, wp, wb = _work(table_grad_work_bytes(n, num_rows, dim), work, device, stream)
    _run("lsmgnn_embed_grad", device, stream, dp, dim, dld, dt, ip, n, num_rows, NO_PAD if pad is None else pad,
         scale, gp, gld, gt, wp, wb, status_ptr)
    return grad


def embed_grad_rows_async(dy, ids, num_rows, unique, rows, result_ptr, scale=1.0, pad=None, work=None, stream=None):
    """Queue the gradient of embed_rows' table by rows (lsmgnn_embed_grad_rows):
    unique (int64, n entries) receives the distinct IDs, ascending, and rows
    (n, dim) their gradients; once `stream` has run it, the two uint64 at
    result_ptr hold how many there are and the status code."""
    import torch
    device = dy.device
    dp, n, dim, dld, dt = _matrix(dy, "dy")
    ip = _vector(ids, torch.int64, n, "ids", device)
    up = _vector(unique, torch.int64, n, "unique", device)
    rp, _, _, rld, rt = _matrix(rows, "rows", dim, n, device)
    work, wp, wb = _work(embed_grad_work_bytes(n, num_rows, dim), work, device, stream)
    _run("lsmgnn_embed_grad_rows", device, stream, dp, dim, dld, dt, ip, n, num_rows, NO_PAD if pad is None else pad,
         scale, up, rp, rld, rt, wp, wb, result_ptr)


def embed_grad_rows(dy, ids, num_rows, scale=1.0, pad=None, dtype=None, work=None, stream=None):
    """The rows of embed_rows' table gradient that are not zero by construction:
    (unique, rows), the distinct IDs ascending and their gradients.  Waits for
    the stream to know how many there are; raises on an ID out of range."""
    import torch
    _matrix(dy, "dy")
    device = dy.device
    n = ids.numel()
    unique = _empty(n, torch.int64, device, stream)
    rows = _empty(tuple(dy.shape), dtype or dy.dtype, device, stream)
    result = torch.empty(2, dtype=torch.int64, pin_memory=True)
    embed_grad_rows_async(dy, ids, num_rows, unique, rows, result.data_ptr(), scale, pad, work, stream)
    (torch.cuda.current_stream(device) if stream is None else stream).synchronize()
    count, status = result.tolist()
    _check(status, "lsmgnn_embed_grad_rows")
    return unique[:count], rows[:count]


class RoutePlan:
    """Where the choices of n tokens go when their rows are sorted by expert:
    offsets (num_experts + 1), slot (n, k) and source (rows), int32 device
    tensors as lsmgnn_route_plan writes them (views of one buffer)."""

    __slots__ = ("n", "k", "num_experts", "align", "rows", "device", "buffer", "_at_slot", "_at_source")

    def __init__(self, n, k, num_experts, align, rows, device, stream):
        import torch
        self.n, self.k, self.num_experts, self.align, self.rows, self.device = n, k, num_experts, align, rows, device
        # the offsets, the slots, the sources, each 16-byte aligned
        self._at_slot = (num_experts + 4) // 4 * 4
        self._at_source = self._at_slot + (n * k + 3) // 4 * 4
        self.buffer = _empty(self._at_source + rows, torch.int32, device, stream)

    @property
    def offsets(self):
        return self.buffer[: self.num_experts + 1]

    @property
    def slot(self):
        return self.buffer[self._at_slot: self._at_slot + self.n * self.k].view(self.n, self.k)

    @property
    def source(self):
        return self.buffer[self._at_source:]

    def _ptrs(self):
        """Addresses of offsets, slot and source."""
        base = self.buffer.data_ptr()
        return base, base + 4 * self._at_slot, base + 4 * self._at_source


def route_plan(experts, num_experts, align=1, work=None, status_ptr=None, stream=None):
    """Plan of the rows sorted by expert (lsmgnn_route_plan) from the choices
    (n, k) int64 (negative: dropped), each expert's rows rounded up to `align`.
    Nothing waits: the offsets stay on the device.  status_ptr: address of a
    uint64 that receives E_RANGE for a choice that is too large."""
    import torch
    ep = _dev_ptr(experts, torch.int64, "experts")
    if experts.dim() != 2:
        raise ValueError("experts must have two dimensions, tokens and choices")
    n, k = experts.shape
    device = experts.device
    L = lib()
    rows = L.lsmgnn_route_max_rows(n, k, num_experts, align)
    if rows >= 1 << 31:
        raise ValueError("too many sorted rows")
    plan = RoutePlan(n, k, num_experts, align, rows, device, stream)
    work, wp, wb = _work(L.lsmgnn_route_work_bytes(n, k, num_experts), work, device, stream)
    _run("lsmgnn_route_plan", device, stream, ep, n, k, num_experts, align, *plan._ptrs(), wp, wb, status_ptr)
    return plan


def route_rows(x, plan, out=None, stream=None):
    """x's rows sorted by expert (lsmgnn_route_rows): (plan.rows, dim), zeros in
    the unused rows."""
    device = x.device
    xp, n, dim, xld, xt = _matrix(x, "x", rows=plan.n, like=plan.device)
    out, op, old, ot = _output(out, "out", plan.rows, dim, x.dtype, device, stream)
    if ot != xt:
        raise TypeError("x and out must have one type")
    _run("lsmgnn_route_rows", device, stream, xp, n, dim, xld, xt, *plan._ptrs()[1:], plan.k, plan.rows, op, old)
    return out


def route_combine(z, plan, weights=None, out=None, stream=None):
    """Sorted rows back to their tokens (lsmgnn_route_combine): out[t] = the sum
    over the kept choices of weights[t, j] * z[slot[t, j]] (weights: (n, k)
    float32, or None for ones: the gradient of route_rows)."""
    import torch
    device = z.device
    zp, rows, dim, zld, zt = _matrix(z, "z", rows=plan.rows, like=plan.device)
    wp = None if weights is None else _vector(weights, torch.float32, plan.n * plan.k, "weights", device, True)
    out, op, old, ot = _output(out, "out", plan.n, dim, z.dtype, device, stream)
    if ot != zt:
        raise TypeError("z and out must have one type")
    _run("lsmgnn_route_combine", device, stream, zp, rows, dim, zld, zt, plan._ptrs()[1], wp, plan.n, plan.k, op, old)
    return out


def route_combine_grad(dy, z, plan, weights, dz=None, stream=None):
    """The gradients of route_combine (lsmgnn_route_combine_grad): (dz, dweights)
    from dy (n, dim), the sorted rows z it combined and its weights (n, k)."""
    import torch
    device = dy.device
    dp, n, dim, dld, dt = _matrix(dy, "dy", rows=plan.n, like=plan.device)
    zp, rows, _, zld, zt = _matrix(z, "z", dim, plan.rows, device)
    wp = _vector(weights, torch.float32, plan.n * plan.k, "weights", device, True)
    dz, op, old, ot = _output(dz, "dz", rows, dim, dy.dtype, device, stream)
    if zt != dt or ot != dt:
        raise TypeError("dy, z and dz must have one type")
    dw = _empty((plan.n, plan.k), torch.float32, device, stream)
    _run("lsmgnn_route_combine_grad", device, stream, dp, n, dim, dld, dt, zp, zld, *plan._ptrs()[1:], wp, plan.k,
         rows, op, old, dw.data_ptr())
    return dz, dw


class Packed8:
    """Rows kept in 8 bits: q (rows, dim) int8 and scale (rows, blocks) uint8,
    a value being q * 2^(scale - 127) with the scale of its block of 32 (views of
    one buffer).  A gated activation's rows come in pairs, one for each half."""

    __slots__ = ("rows", "dim", "blocks", "device", "buffer", "_at_scale")

    def __init__(self, rows, dim, device, stream=None):
        import torch
        self.rows, self.dim, self.blocks = rows, dim, (dim + PACK_BLOCK - 1) // PACK_BLOCK
        self._at_scale = (rows * dim + 255) // 256 * 256
        self.buffer = _empty(self._at_scale + rows * self.blocks, torch.uint8, device, stream)
        self.device = self.buffer.device

    @property
    def q(self):
        import torch
        return self.buffer[: self.rows * self.dim].view(torch.int8).view(self.rows, self.dim)

    @property
    def scale(self):
        return self.buffer[self._at_scale:].view(self.rows, self.blocks)

    def _ptrs(self, rows, dim, device):
        """Addresses of q and scale, for rows of `dim`."""
        if (rows, dim) != (self.rows, self.dim):
            raise ValueError(f"packed must hold {rows} rows of {dim}, not {self.rows} of {self.dim}")
        if device != self.device:
            raise ValueError(f"packed is on {self.device}, not on {device}")
        base = self.buffer.data_ptr()
        return base, base + self._at_scale


def _act_code(act):
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, not {act!r}")
    return ACTIVATIONS[act]


def pack8(x, packed=None, stream=None):
    """x (rows, dim) kept in 8 bits (lsmgnn_pack8)."""
    device = x.device
    xp, rows, dim, ld, t = _matrix(x, "x")
    packed = packed or Packed8(rows, dim, device, stream)
    qp, sp = packed._ptrs(rows, dim, device)
    _run("lsmgnn_pack8", device, stream, xp, rows, dim, ld, t, qp, sp)
    return packed


def unpack8(packed, dtype=None, out=None, stream=None):
    """The kept values (lsmgnn_unpack8) as `dtype` (default bfloat16, which holds
    them exactly)."""
    import torch
    device, rows, dim = packed.device, packed.rows, packed.dim
    out, op, ld, t = _output(out, "out", rows, dim, dtype or torch.bfloat16, device, stream)
    qp, sp = packed._ptrs(rows, dim, device)
    _run("lsmgnn_unpack8", device, stream, qp, sp, rows, dim, op, ld, t)
    return out


def act8(x, act, gated=False, out=None, packed=None, stream=None):
    """An activation and what its backward pass keeps (lsmgnn_act8): (y, packed)
    with y = f(x), or gated y = f(a) * b for x = [a | b]; act: a name in
    ACTIVATIONS."""
    device = x.device
    code, parts = _act_code(act), 2 if gated else 1
    xp, rows, width, ld, t = _matrix(x, "x")
    dim = width // parts
    if dim * parts != width:
        raise ValueError("a gated activation's input must have an even width")
    out, yp, yld, yt = _output(out, "out", rows, dim, x.dtype, device, stream)
    if yt != t:
        raise TypeError("x and out must have one type")
    packed = packed or Packed8(rows * parts, dim, device, stream)
    qp, sp = packed._ptrs(rows * parts, dim, device)
    _run("lsmgnn_act8", device, stream, xp, rows, dim, ld, t, code, parts - 1, yp, yld, qp, sp)
    return out, packed


def act8_grad(dy, packed, act, gated=False, dx=None, stream=None):
    """act8's gradient with respect to x from dy and the kept values
    (lsmgnn_act8_grad): (rows, dim), or gated (rows, 2 dim)."""
    device = dy.device
    code, parts = _act_code(act), 2 if gated else 1
    dp, rows, dim, dld, t = _matrix(dy, "dy")
    dx, xp, xld, xt = _output(dx, "dx", rows, dim * parts, dy.dtype, device, stream)
    if xt != t:
        raise TypeError("dy and dx must have one type")
    qp, sp = packed._ptrs(rows * parts, dim, device)
    _run("lsmgnn_act8_grad", device, stream, dp, rows, dim, dld, t, qp, sp, code, parts - 1, xp, xld)
    return dx


def weight_grad8_work_bytes(rows, din, dout, num_experts=1):
    """Device work memory weight_grad8 needs."""
    return int(lib().lsmgnn_weight_grad8_work_bytes(int(rows), int(din), int(dout), int(num_experts)))


def weight_grad8(packed, dy, offsets=None, dtype=None, out=None, work=None, stream=None):
    """Weight gradients of products whose input was kept in 8 bits
    (lsmgnn_weight_grad8): (num_experts, din, dout) float32 (or `dtype`), expert
    e's from the rows [offsets[e], offsets[e + 1]) of packed and dy (rows, dout);
    offsets: num_experts + 1 int32 on the device (a plan's), or None for one
    expert with all rows."""
    import torch
    device = dy.device
    dp, rows, dout, dld, dt = _matrix(dy, "dy")
    din = packed.dim
    qp, sp = packed._ptrs(rows, din, device)
    experts = 1 if offsets is None else offsets.numel() - 1
    fp = None if offsets is None else _vector(offsets, torch.int32, experts + 1, "offsets", device)
    if out is None:
        out = _empty((experts, din, dout), dtype or torch.float32, device, stream)
    op = _vector(out, out.dtype, experts * din * dout, "out", device, True)
    work, wp, wb = _work(weight_grad8_work_bytes(rows, din, dout, experts), work, device, stream)
    _run("lsmgnn_weight_grad8", device, stream, qp, sp, rows, din, dp, dout, dld, dt, fp, experts, op,
         _type_code(out.dtype, "out"), wp, wb)
    return out
