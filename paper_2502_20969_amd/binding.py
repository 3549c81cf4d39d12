"""ctypes binding of libivf.so: same names as include/ivf.h, argument marshalling only.

Host arguments are numpy arrays (or CPU torch tensors); device arguments are torch CUDA
tensors.  Nothing here computes: every step of the search runs in the HIP library, and the
module raises at import of the library if it has not been built.
"""
import collections
import ctypes as C
import functools
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libivf.so")

IVF_IP, IVF_L2 = 0, 1
IVF_F32, IVF_F16, IVF_BF16, IVF_E4M3 = 0, 1, 2, 3
IVF_PLACE_DEVICE, IVF_PLACE_HOST = 0, 1
IVF_PREFETCH_RESET = 1
IVF_MAX_K = 112
IVF_MAX_BEAMS, IVF_MAX_BEAM_STATES = 64, 8
DTYPE_CODE = {"f32": IVF_F32, "f16": IVF_F16, "bf16": IVF_BF16}

EXPORTS = [
    "ivf_build_layout", "ivf_adopt_layout", "ivf_free", "ivf_prefetch", "ivf_prefetch_wait",
    "ivf_search", "ivf_search_device", "ivf_search_device_noalloc", "ivf_reserve", "ivf_coarse_scores", "ivf_probe",
    "ivf_prefetch_ways", "ivf_resident", "ivf_batched_scores", "ivf_get_layout", "ivf_profile_enable", "ivf_profile_read",
    "ivf_profile_reset", "ivf_set_host_threads", "ivf_set_pipeline_depth", "ivf_synchronize",
    "ivf_set_batch_mode", "ivf_limit_batch_memory", "ivf_cache_configure", "ivf_cache_end_round", "ivf_cache_hotness",
    "ivf_schedule", "ivf_kv_append", "ivf_attend", "ivf_attend_workspace", "ivf_kv_read", "ivf_verify_draft", "ivf_verify_workspace", "ivf_beam_step", "ivf_beam_workspace", "ivf_host_scan", "ivf_host_scan_capacity", "ivf_prefetch_amount", "ivf_prefetch_plan", "ivf_cache_plan", "ivf_strerror", "ivf_last_error",
]


class CacheStats(C.Structure):
    _fields_ = [("n_cached", C.c_int32), ("n_evicted", C.c_int32), ("bytes_cached", C.c_uint64),
                ("bytes_kept", C.c_uint64), ("bytes_moved", C.c_uint64), ("ms_update", C.c_float),
                ("ms_compact", C.c_float), ("n_launches", C.c_int32)]


class PrefetchStats(C.Structure):
    _fields_ = [("n_ranked", C.c_int32), ("n_taken", C.c_int32), ("n_skipped", C.c_int32),
                ("n_resident", C.c_int32), ("bytes", C.c_uint64), ("buffer_used", C.c_uint64)]


class SearchStats(C.Structure):
    _fields_ = [("n_probed", C.c_int32), ("n_overlap", C.c_int32), ("n_miss", C.c_int32),
                ("hit_rate", C.c_float), ("bytes_gpu", C.c_uint64), ("bytes_host", C.c_uint64),
                ("ms_total", C.c_float), ("ms_probe", C.c_float), ("ms_host_scan", C.c_float),
                ("n_exact_gpu", C.c_int32), ("n_exact_host", C.c_int32)]


class Profile(C.Structure):
    _fields_ = [("calls", C.c_uint64), ("ms_coarse", C.c_double), ("ms_select", C.c_double),
                ("ms_scan", C.c_double), ("ms_merge", C.c_double), ("scan_bytes", C.c_uint64),
                ("scan_rows", C.c_uint64)]


class KvCacheArg(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int64), ("page_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("page", C.c_int32), ("n_heads", C.c_int32),
                ("d", C.c_int32), ("dtype", C.c_int32), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("scale_page_stride", C.c_int64), ("scale_token_stride", C.c_int64), ("scale_head_stride", C.c_int64), ("row_dtype", C.c_int32)]


class KvStepArg(C.Structure):
    _fields_ = [("q_off", C.c_void_p), ("len", C.c_void_p), ("table", C.c_void_p), ("table_stride", C.c_int64),
                ("group_off", C.c_void_p), ("prefix_len", C.c_void_p), ("prefix_table", C.c_void_p), ("prefix_stride", C.c_int64),
                ("n_seq", C.c_int32), ("n_tokens", C.c_int32), ("page", C.c_int32), ("max_q", C.c_int32), ("max_len", C.c_int32),
                ("n_groups", C.c_int32), ("prefix_page", C.c_int32), ("max_prefix", C.c_int32)]


class RowsArg(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class BeamStateArg(C.Structure):
    _fields_ = [("from_", C.c_void_p), ("to", C.c_void_p), ("row_bytes", C.c_int64), ("from_stride", C.c_int64),
                ("to_stride", C.c_int64)]


class IvfError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"libivf status {status}: {text}")
        self.status = status


_lib = None


def load():
    """Loads libivf.so; fails loudly when it is missing (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, sz, u32, ci = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_uint32, C.c_int
    L.ivf_build_layout.argtypes = [vp, i64, i32, ci, vp, i32, vp, vp, ci, ci, sz, vp, vp, C.POINTER(vp)]
    L.ivf_adopt_layout.argtypes = [vp, vp, vp, i64, i32, ci, vp, i32, ci, ci, sz, vp, vp, C.POINTER(vp)]
    L.ivf_free.argtypes = [vp]
    L.ivf_free.restype = None
    L.ivf_prefetch.argtypes = [vp, vp, i32, i32, sz, u32, C.POINTER(PrefetchStats)]
    L.ivf_prefetch_wait.argtypes = [vp, C.POINTER(C.c_float)]
    L.ivf_prefetch_ways.argtypes = [vp, C.POINTER(i32), C.POINTER(i32)]
    L.ivf_search.argtypes = [vp, vp, i32, i32, i32, vp, vp, C.POINTER(SearchStats)]
    L.ivf_search_device.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    L.ivf_search_device_noalloc.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    L.ivf_reserve.argtypes = [vp, i32, i32, i32]
    L.ivf_coarse_scores.argtypes = [vp, vp, i32, vp]
    L.ivf_probe.argtypes = [vp, vp, i32, i32, vp]
    L.ivf_resident.argtypes = [vp, vp, C.POINTER(i32)]
    L.ivf_batched_scores.argtypes = [vp, vp, i32, i32, vp, vp]
    L.ivf_get_layout.argtypes = [vp, vp, vp]
    L.ivf_profile_enable.argtypes = [vp, ci]
    L.ivf_profile_read.argtypes = [vp, C.POINTER(Profile)]
    L.ivf_profile_reset.argtypes = [vp]
    L.ivf_set_host_threads.argtypes = [vp, i32]
    L.ivf_set_pipeline_depth.argtypes = [vp, i32]
    L.ivf_synchronize.argtypes = [vp]
    L.ivf_set_batch_mode.argtypes = [vp, i32]
    L.ivf_limit_batch_memory.argtypes = [vp, sz]
    L.ivf_cache_configure.argtypes = [vp, C.c_float, C.c_float, C.c_float, C.c_float]
    L.ivf_cache_end_round.argtypes = [vp, C.POINTER(CacheStats)]
    L.ivf_cache_hotness.argtypes = [vp, vp]
    L.ivf_schedule.argtypes = [vp, vp, i32, i32, vp, C.POINTER(C.c_float)]
    step, cache, rows = C.POINTER(KvStepArg), C.POINTER(KvCacheArg), C.POINTER(RowsArg)
    L.ivf_kv_append.argtypes = [step, cache, rows, rows, vp, i32, i32, i32, vp, rows, rows, i32, vp]
    L.ivf_attend_workspace.argtypes = [step, cache, i32, i32, i32, C.POINTER(sz)]
    L.ivf_attend.argtypes = [step, cache, rows, i32, rows, vp, C.c_float, i32, i32, vp, sz, vp]
    L.ivf_kv_read.argtypes = [step, cache, vp, vp, i64, rows, rows, vp]
    L.ivf_verify_workspace.argtypes = [i32, i32, i32, C.POINTER(sz)]
    L.ivf_verify_draft.argtypes = [step, vp, i64, ci, i32, C.c_double, vp, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    L.ivf_beam_workspace.argtypes = [i32, i32, i32, i32, C.POINTER(sz)]
    L.ivf_beam_step.argtypes = [vp, i64, ci, i32, i32, i32, vp, vp, i32, i32, vp, vp, vp, vp, C.POINTER(BeamStateArg), i32, vp, sz, vp]
    L.ivf_strerror.argtypes = [ci]
    L.ivf_strerror.restype = C.c_char_p
    L.ivf_last_error.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("ivf_free", "ivf_strerror", "ivf_last_error"):
            getattr(L, name).restype = ci
    _lib = L
    return L


_torch_mod = None


def _torch():
    global _torch_mod
    if _torch_mod is None:
        import torch
        _torch_mod = torch
    return _torch_mod


def _check(status):
    if status != 0:
        L = load()
        raise IvfError(status, f"{L.ivf_strerror(status).decode()} ({L.ivf_last_error().decode()})")


def _host(a, dtype):
    """numpy view of a host array in the dtype the ABI wants (no arithmetic, copies only if needed)."""
    if a is None:
        return None
    if hasattr(a, "detach"):          # torch CPU tensor
        assert a.device.type == "cpu", "expected a host array"
        import torch
        if a.dtype == torch.bfloat16:
            a = a.contiguous().view(torch.int16)
        a = a.detach().contiguous().numpy()
    if dtype is None:
        return np.ascontiguousarray(a)
    return np.ascontiguousarray(a, dtype=dtype)


def _ptr(a):
    if a is None:
        return None
    if hasattr(a, "data_ptr"):
        return C.c_void_p(a.data_ptr())
    return C.c_void_p(a.ctypes.data)


def _stream(s):
    return None if s is None else C.c_void_p(s.cuda_stream)


def _rows_host(vectors, dtype):
    code = DTYPE_CODE[dtype]
    if code == IVF_F32:
        return _host(vectors, np.float32)
    a = _host(vectors, None)
    if a.dtype == np.float16:
        a = a.view(np.uint16)
    if a.dtype == np.int16:
        a = a.view(np.uint16)
    assert a.dtype == np.uint16 and a.flags["C_CONTIGUOUS"]
    return a


class Index:
    """Owner of one ivf_index handle."""

    def __init__(self, handle, d, nlist, n, keep=()):
        self._h = handle
        self.d, self.nlist, self.n = d, nlist, n
        self._keep = keep      # arrays the index adopted and that must outlive it
        # device tensors of searches the library may still touch (a pipelined or list-major call is
        # finished when its stream is next needed or in ivf_synchronize): one entry per stream at most
        self._inflight = collections.deque(maxlen=32)
        self._search_device = load().ivf_search_device
        t = _torch()
        self._f32, self._i64 = t.float32, t.int64

    def _device_triple(self, q_dev, k, ids_dev, dists_dev):
        """Checks the three device tensors of a device-side search (this runs once per search: kept short);
        returns the number of queries."""
        if q_dev.dtype is not self._f32 or ids_dev.dtype is not self._i64 or dists_dev.dtype is not self._f32:
            raise TypeError("queries and distances must be float32, ids int64")
        if not (q_dev.is_cuda and ids_dev.is_cuda and dists_dev.is_cuda):
            raise ValueError("expected CUDA tensors")
        if not (q_dev.is_contiguous() and ids_dev.is_contiguous() and dists_dev.is_contiguous()):
            raise ValueError("expected contiguous tensors")
        nq = q_dev.numel() // self.d
        if ids_dev.numel() < nq * k or dists_dev.numel() < nq * k:
            raise ValueError("ids / dists hold fewer than nq * k entries")
        return nq

    def close(self):
        if self._h is not None:
            load().ivf_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- lookahead -------------------------------------------------------------------------
    def ivf_prefetch(self, q_in, nprobe, budget_bytes, flags=0):
        q = _host(q_in, np.float32).reshape(-1, self.d)
        st = PrefetchStats()
        _check(load().ivf_prefetch(self._h, _ptr(q), q.shape[0], nprobe, int(budget_bytes), flags, C.byref(st)))
        return st

    def ivf_prefetch_wait(self):
        ms = C.c_float(0)
        _check(load().ivf_prefetch_wait(self._h, C.byref(ms)))
        return ms.value

    # -- search ------------------------------------------------------------------------------
    def ivf_prefetch_ways(self):
        by_kernel, by_engine = C.c_int32(), C.c_int32()
        _check(load().ivf_prefetch_ways(self._h, C.byref(by_kernel), C.byref(by_engine)))
        return by_kernel.value, by_engine.value

    def ivf_search(self, q_out, nprobe, k, with_stats=False):
        q = _host(q_out, np.float32).reshape(-1, self.d)
        nq = q.shape[0]
        ids = np.empty((nq, k), dtype=np.int64)
        dists = np.empty((nq, k), dtype=np.float32)
        st = SearchStats()
        _check(load().ivf_search(self._h, _ptr(q), nq, nprobe, k, _ptr(ids), _ptr(dists), C.byref(st)
                                 if with_stats else None))
        return (ids, dists, st) if with_stats else (ids, dists)

    def ivf_search_device(self, q_dev, nprobe, k, ids_dev, dists_dev):
        """q_dev [nq, d] float32, ids_dev [nq, k] int64, dists_dev [nq, k] float32: CUDA tensors.
        The three tensors are kept referenced until ivf_synchronize (the library may read the queries
        and rewrite the outputs until then)."""
        nq = self._device_triple(q_dev, k, ids_dev, dists_dev)
        self._inflight.append((q_dev, ids_dev, dists_dev))
        status = self._search_device(self._h, q_dev.data_ptr(), nq, nprobe, k, ids_dev.data_ptr(), dists_dev.data_ptr())
        if status != 0:
            _check(status)

    def ivf_search_device_noalloc(self, q_dev, nprobe, k, ids_dev, dists_dev):
        """ivf_search_device on the library's fixed scratch area: allocates nothing."""
        nq = self._device_triple(q_dev, k, ids_dev, dists_dev)
        _check(load().ivf_search_device_noalloc(self._h, _ptr(q_dev), nq, nprobe, k, _ptr(ids_dev), _ptr(dists_dev)))

    def ivf_reserve(self, nq, nprobe, k):
        _check(load().ivf_reserve(self._h, nq, nprobe, k))

    # -- stages ------------------------------------------------------------------------------
    def ivf_coarse_scores(self, q):
        q = _host(q, np.float32).reshape(-1, self.d)
        out = np.empty((q.shape[0], self.nlist), dtype=np.float64)
        _check(load().ivf_coarse_scores(self._h, _ptr(q), q.shape[0], _ptr(out)))
        return out

    def ivf_probe(self, q, nprobe):
        q = _host(q, np.float32).reshape(-1, self.d)
        out = np.empty((q.shape[0], min(nprobe, self.nlist)), dtype=np.int32)
        _check(load().ivf_probe(self._h, _ptr(q), q.shape[0], nprobe, _ptr(out)))
        return out

    def ivf_batched_scores(self, q, cluster, rows_in_cluster):
        """MFMA filter scores [nq, rows] of one cluster and the error bound eps [nq] the scan assumes."""
        q = _host(q, np.float32).reshape(-1, self.d)
        scores = np.empty((q.shape[0], rows_in_cluster), dtype=np.float32)
        eps = np.empty(q.shape[0], dtype=np.float32)
        _check(load().ivf_batched_scores(self._h, _ptr(q), q.shape[0], int(cluster), _ptr(scores), _ptr(eps)))
        return scores, eps

    def ivf_resident(self):
        n = C.c_int32(self.nlist)
        out = np.empty(self.nlist, dtype=np.int32)
        _check(load().ivf_resident(self._h, _ptr(out), C.byref(n)))
        return out[:n.value].copy()

    def ivf_get_layout(self):
        off = np.empty(self.nlist + 1, dtype=np.int64)
        ids = np.empty(self.n, dtype=np.int64)
        _check(load().ivf_get_layout(self._h, _ptr(off), _ptr(ids)))
        return off, ids

    # -- prefetching scheduler ---------------------------------------------------------------
    def ivf_schedule(self, q, micro, with_time=False):
        q = _host(q, np.float32).reshape(-1, self.d)
        order = np.empty(q.shape[0], dtype=np.int32)
        ms = C.c_float(0)
        _check(load().ivf_schedule(self._h, _ptr(q), q.shape[0], int(micro), _ptr(order), C.byref(ms)))
        return (order, ms.value) if with_time else order

    # -- cluster cache -----------------------------------------------------------------------
    def ivf_cache_configure(self, fraction=0.5, h_init=1.0, decay=2.0, h_inc=1.0):
        _check(load().ivf_cache_configure(self._h, C.c_float(fraction), C.c_float(h_init), C.c_float(decay),
                                          C.c_float(h_inc)))

    def ivf_cache_end_round(self):
        st = CacheStats()
        _check(load().ivf_cache_end_round(self._h, C.byref(st)))
        return st

    def ivf_cache_hotness(self):
        out = np.empty(self.nlist, dtype=np.float32)
        _check(load().ivf_cache_hotness(self._h, _ptr(out)))
        return out

    # -- profiling ---------------------------------------------------------------------------
    def ivf_profile_enable(self, on=True):
        _check(load().ivf_profile_enable(self._h, 1 if on else 0))

    def ivf_profile_read(self):
        p = Profile()
        _check(load().ivf_profile_read(self._h, C.byref(p)))
        return p

    def ivf_profile_reset(self):
        _check(load().ivf_profile_reset(self._h))

    def ivf_set_host_threads(self, n):
        _check(load().ivf_set_host_threads(self._h, n))

    def ivf_set_pipeline_depth(self, depth):
        _check(load().ivf_set_pipeline_depth(self._h, depth))

    def ivf_synchronize(self):
        _check(load().ivf_synchronize(self._h))
        self._inflight.clear()

    def ivf_set_batch_mode(self, mode):
        _check(load().ivf_set_batch_mode(self._h, mode))

    def ivf_limit_batch_memory(self, limit):
        _check(load().ivf_limit_batch_memory(self._h, limit))


def ivf_build_layout(vectors, dtype, centroids, assign, ids=None, metric=IVF_IP,
                     placement=IVF_PLACE_DEVICE, device_buffer_bytes=0, compute_stream=None,
                     copy_stream=None):
    rows = _rows_host(vectors, dtype)
    cent = _host(centroids, np.float32)
    asg = _host(assign, np.int32)
    idv = _host(ids, np.int64)
    n, d = rows.shape
    nlist = cent.shape[0]
    assert cent.shape[1] == d and asg.shape[0] == n
    h = C.c_void_p()
    _check(load().ivf_build_layout(_ptr(rows), n, d, DTYPE_CODE[dtype], _ptr(cent), nlist, _ptr(asg),
                                   _ptr(idv), metric, placement, int(device_buffer_bytes),
                                   _stream(compute_stream), _stream(copy_stream), C.byref(h)))
    return Index(h, d, nlist, n)


def ivf_adopt_layout(lists, dtype, offsets, centroids, ids=None, metric=IVF_IP,
                     placement=IVF_PLACE_DEVICE, device_buffer_bytes=0, compute_stream=None,
                     copy_stream=None):
    """lists: torch tensor [n, d], on the GPU (device placement) or pinned on the host."""
    assert lists.is_contiguous()
    if placement == IVF_PLACE_DEVICE:
        assert lists.is_cuda
    else:
        assert (not lists.is_cuda) and lists.is_pinned()
    n, d = lists.shape
    cent = _host(centroids, np.float32)
    off = _host(offsets, np.int64)
    idv = _host(ids, np.int64)
    nlist = cent.shape[0]
    h = C.c_void_p()
    _check(load().ivf_adopt_layout(_ptr(lists), _ptr(off), _ptr(idv), n, d, DTYPE_CODE[dtype], _ptr(cent),
                                   nlist, metric, placement, int(device_buffer_bytes),
                                   _stream(compute_stream), _stream(copy_stream), C.byref(h)))
    return Index(h, d, nlist, n, keep=(lists,))


def ivf_host_scan(lists, dtype, offsets, q, clusters, k, ids=None, metric=IVF_IP, threads=4):
    """Host scan of the listed clusters for one query: (ids, float64 scores) of the candidates the
    merge step would receive, unordered.  lists: host array [n, d] in the stored type."""
    rows = _rows_host(lists, dtype)
    off = _host(offsets, np.int64)
    idv = _host(ids, np.int64)
    qv = _host(q, np.float32).reshape(-1)
    cl = _host(clusters, np.int32).reshape(-1)
    d = rows.shape[1]
    assert qv.shape[0] == d
    L = load()
    cap = max(1, int(L.ivf_host_scan_capacity(int(k))))      # 0 for a k the library will refuse below
    out_ids = np.empty(cap, dtype=np.int64)
    out_scores = np.empty(cap, dtype=np.float64)
    n_out = C.c_int32(0)
    _check(L.ivf_host_scan(_ptr(rows), _ptr(off), _ptr(idv), d, DTYPE_CODE[dtype], metric, _ptr(qv), _ptr(cl),
                           cl.shape[0], k, threads, _ptr(out_ids), _ptr(out_scores), C.byref(n_out)))
    return out_ids[:n_out.value], out_scores[:n_out.value]


def ivf_prefetch_amount(bandwidth, t_llm, nprobe, t_cc, budgets, miss_rates):
    """The prefetch budget of App. C for a measured miss-rate curve: (bytes, seconds of t_1 + t_2, case)."""
    bs = _host(budgets, np.float64).reshape(-1)
    rs = _host(miss_rates, np.float64).reshape(-1)
    assert bs.shape == rs.shape
    L = load()
    L.ivf_prefetch_amount.argtypes = [C.c_double, C.c_double, C.c_int32, C.c_double, C.c_void_p, C.c_void_p, C.c_int32,
                                      C.c_void_p, C.c_void_p, C.c_void_p]
    amount, seconds, which = C.c_double(0.0), C.c_double(0.0), C.c_int32(0)
    _check(L.ivf_prefetch_amount(float(bandwidth), float(t_llm), int(nprobe), float(t_cc), _ptr(bs), _ptr(rs), bs.shape[0],
                                 C.byref(amount), C.byref(seconds), C.byref(which)))
    return amount.value, seconds.value, which.value


def ivf_prefetch_plan(ranked, offsets, row_bytes, budget_bytes, buffer_bytes, resident_off, buffer_used):
    """The budget walk of ivf_prefetch over already ranked clusters (ranked: [nq, nprobe] int32).
    resident_off (int64[nlist], -1 = absent) is updated in place.  Returns (clusters to copy in
    order, PrefetchStats, buffer bytes in use afterwards)."""
    rk = _host(ranked, np.int32)
    rk = rk.reshape(1, -1) if rk.ndim == 1 else rk
    off = _host(offsets, np.int64)
    assert resident_off.dtype == np.int64 and resident_off.flags["C_CONTIGUOUS"]
    nlist = off.shape[0] - 1
    assert resident_off.shape[0] == nlist
    taken = np.empty(rk.size, dtype=np.int32)
    n_taken = C.c_int32(0)
    used = C.c_size_t(int(buffer_used))
    st = PrefetchStats()
    L = load()
    L.ivf_prefetch_plan.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_size_t, C.c_size_t,
                                    C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    _check(L.ivf_prefetch_plan(_ptr(rk), rk.shape[0], rk.shape[1], _ptr(off), nlist, int(row_bytes), int(budget_bytes),
                               int(buffer_bytes), _ptr(resident_off), C.byref(used), _ptr(taken), C.byref(n_taken),
                               C.byref(st)))
    return taken[:n_taken.value], st, used.value


class CacheMove(C.Structure):
    _fields_ = [("cluster", C.c_int32), ("via_staging", C.c_int32), ("from_byte", C.c_uint64),
                ("to_byte", C.c_uint64), ("bytes", C.c_uint64)]


def ivf_cache_plan(hotness, offsets, row_bytes, resident_off, buffer_used, buffer_bytes, fraction):
    """Eviction and consolidation plan of a cache round.  hotness (float32[nlist]) and resident_off
    (int64[nlist]) are updated in place.  Returns (evicted clusters in order, list of moves as
    (cluster, via_staging, from_byte, to_byte, bytes), buffer bytes in use afterwards)."""
    assert hotness.dtype == np.float32 and hotness.flags["C_CONTIGUOUS"]
    assert resident_off.dtype == np.int64 and resident_off.flags["C_CONTIGUOUS"]
    off = _host(offsets, np.int64)
    nlist = off.shape[0] - 1
    assert hotness.shape[0] == nlist and resident_off.shape[0] == nlist
    evicted = np.empty(nlist, dtype=np.int32)
    moves = (CacheMove * nlist)()
    n_ev, n_mv = C.c_int32(0), C.c_int32(0)
    used = C.c_size_t(int(buffer_used))
    L = load()
    L.ivf_cache_plan.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_size_t, C.c_void_p, C.c_void_p, C.c_size_t,
                                 C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    _check(L.ivf_cache_plan(_ptr(hotness), _ptr(off), nlist, int(row_bytes), _ptr(resident_off), C.byref(used),
                            int(buffer_bytes), float(fraction), _ptr(evicted), C.byref(n_ev), moves, C.byref(n_mv)))
    mv = [(m.cluster, m.via_staging, m.from_byte, m.to_byte, m.bytes) for m in moves[:n_mv.value]]
    return evicted[:n_ev.value], mv, used.value


# ---- answering from retrieved passages -------------------------------------------------------------
_codes = None


def _code(dtype):
    global _codes
    if _codes is None:
        t = _torch()
        _codes = {t.float32: IVF_F32, t.float16: IVF_F16, t.bfloat16: IVF_BF16}
    code = _codes.get(dtype)
    if code is None:
        raise TypeError(f"{dtype}: float32, float16 or bfloat16 expected")
    return code


def _elsewhere(what, a, device):
    where = f"device {device}" if device >= 0 else "a CUDA device"
    return ValueError(f"{what} is on {a.device}, not on {where} like the rest of the call")


def _i32(a, shape, device, what):
    """A contiguous int32 tensor of this shape (None in it: any size) on this device."""
    t = _torch()
    if a.dtype is not t.int32:
        raise TypeError(f"{what} must be int32")
    if a.get_device() != device or device < 0:
        raise _elsewhere(what, a, device)
    if not a.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if len(a.shape) != len(shape) or any(n is not None and n != m for n, m in zip(shape, a.shape)):
        raise ValueError(f"{what} has shape {tuple(a.shape)}, expected {tuple(shape)}")
    return a.data_ptr()


# The calls below run once per layer and step: their checks are kept short.
def _rows(a, n_tokens, n_heads, cache, what):
    """[n_tokens, n_heads, d] with the elements of a head side by side."""
    if a.dtype is not cache.dtype:
        raise TypeError(f"{what} is {a.dtype}, the cache's rows are {cache.dtype}")
    stride = a.stride()
    if a.shape != (n_tokens, n_heads, cache.d):
        raise ValueError(f"{what} has shape {tuple(a.shape)}, expected [{n_tokens}, {n_heads}, {cache.d}]")
    if a.get_device() != cache.device:
        raise _elsewhere(what, a, cache.device)
    if stride[2] != 1:
        raise ValueError(f"the elements of a head of {what} must lie side by side")
    return RowsArg(a.data_ptr(), stride[0], stride[1])


_byte_types = None


def _bytes(a, codes):
    """Whether a holds e4m3 numbers (codes), or powers of two, in a type of their own or as bytes."""
    global _byte_types
    if _byte_types is None:
        t = _torch()
        _byte_types = (t.uint8, t.float8_e8m0fnu), (t.uint8, t.float8_e4m3fn)
    return a.dtype in _byte_types[codes]


class KvCache:
    """The paged cache of one layer: k and v [n_pages, page, heads, d], views of any page, token and head order
    (a cache of head-major pages is passed as `pages.transpose(1, 2)`).  A quantised cache has e4m3 numbers (float8_e4m3fn or
    uint8) in k and v, their powers of two (float8_e8m0fnu or uint8) in k_scale and v_scale [n_pages, page, heads], in any order,
    and rows of type dtype (float16 or bfloat16)."""

    def __init__(self, k, v, k_scale=None, v_scale=None, dtype=None):
        if k.dtype is not v.dtype or k.shape != v.shape or k.stride() != v.stride():
            raise ValueError("k and v must have the same type, shape and strides")
        if not (k.is_cuda and v.is_cuda) or k.dim() != 4 or k.stride(3) != 1:
            raise ValueError("expected CUDA tensors [n_pages, page, heads, d] with the elements of a head side by side")
        self.k, self.v, self.dtype, self.device = k, v, k.dtype, k.get_device()
        if v.get_device() != self.device:
            raise _elsewhere("v", v, self.device)
        (self.pages, self.page, self.heads, self.d), st = k.shape, k.stride()
        self.k_scale, self.v_scale, self.quantised = k_scale, v_scale, k_scale is not None
        if (k_scale is None) != (v_scale is None) or (k_scale is None) != (dtype is None):
            raise ValueError("k_scale, v_scale and dtype go together")
        if not self.quantised:
            self.arg = KvCacheArg(k.data_ptr(), v.data_ptr(), self.pages, st[0], st[1], st[2], self.page, self.heads, self.d, _code(k.dtype))
        else:
            if not _bytes(k, True) or k_scale.dtype is not v_scale.dtype or not _bytes(k_scale, False):
                raise TypeError("a quantised cache has float8_e4m3fn or uint8 numbers, and float8_e8m0fnu or uint8 scales")
            for what, a in (("k_scale", k_scale), ("v_scale", v_scale)):
                if a.get_device() != self.device:
                    raise _elsewhere(what, a, self.device)
            if k_scale.shape != k.shape[:3] or v_scale.shape != k.shape[:3] or k_scale.stride() != v_scale.stride():
                raise ValueError("expected k_scale and v_scale [n_pages, page, heads] with the same strides")
            self.dtype, sc = dtype, k_scale.stride()
            self.arg = KvCacheArg(k.data_ptr(), v.data_ptr(), self.pages, st[0], st[1], st[2], self.page, self.heads, self.d, IVF_E4M3,
                                  k_scale.data_ptr(), v_scale.data_ptr(), sc[0], sc[1], sc[2], _code(dtype))
        self.ref = C.byref(self.arg)


class KvStep:
    """The sequences of one step, for the calls of all layers.  q_off [sequences + 1], lens [sequences] and table
    [sequences, entries] are int32 CUDA tensors; a table entry names `page` slots.  With group_off [groups + 1]
    the sequences of a group share the prefix of prefix_lens [groups] keys in the rows of prefix_table [groups,
    entries], whose entries name prefix_page slots (default: page).  max_q, max_len and max_prefix are what the
    program knows of the lengths (0: nothing).  The tensors' contents may change between calls."""

    def __init__(self, q_off, lens, table, page, n_tokens, max_q=0, max_len=0, group_off=None, prefix_lens=None, prefix_table=None,
                 prefix_page=None, max_prefix=0):
        n, dev = lens.shape[0], lens.get_device()
        a = KvStepArg(_i32(q_off, (n + 1,), dev, "q_off"), _i32(lens, (n,), dev, "lens"), _i32(table, (n, None), dev, "table"), table.shape[1])
        a.n_seq, a.n_tokens, a.page, a.max_q, a.max_len = n, n_tokens, page, max_q, max_len
        if (group_off is None) != (prefix_lens is None) or (group_off is None) != (prefix_table is None):
            raise ValueError("group_off, prefix_lens and prefix_table go together")
        if group_off is not None:
            g = prefix_lens.shape[0]
            a.group_off, a.prefix_len = _i32(group_off, (g + 1,), dev, "group_off"), _i32(prefix_lens, (g,), dev, "prefix_lens")
            a.prefix_table, a.prefix_stride = _i32(prefix_table, (g, None), dev, "prefix_table"), prefix_table.shape[1]
            a.n_groups, a.prefix_page, a.max_prefix = g, page if prefix_page is None else prefix_page, max_prefix
        self.arg, self.n_tokens, self.device = a, n_tokens, dev
        self._keep = (q_off, lens, table, group_off, prefix_lens, prefix_table)
        self._need = {}            # bytes of workspace by what they depend on
        self.ref = C.byref(a)


def _new(stream, shape, dtype, kept=True):
    """A tensor that the call's kernels on `stream` may write at once (memory that torch last gave to the current stream may
    still be used there); kept: it is for the caller, whose current stream may read it later."""
    t = _torch()
    if stream is None:
        return t.empty(shape, dtype=dtype, device="cuda")
    now = t.cuda.current_stream()
    with t.cuda.stream(stream):
        x = t.empty(shape, dtype=dtype, device="cuda")
    if kept:
        x.record_stream(now)
    return x


def _workspace(n, stream):
    """n bytes that are free again, in stream order, once the call's kernels have run."""
    return _new(stream, n, _torch().uint8, False)


def _room(workspace, device):
    """Place and bytes of the caller's workspace."""
    if workspace.get_device() != device:
        raise _elsewhere("workspace", workspace, device)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace.data_ptr(), workspace.nbytes


_raw_stream = _device_now = None


def _on(stream, device):
    """The stream's handle; None: torch's current one.  Kernels are launched on the current device, which the call's tensors have to be on."""
    global _raw_stream, _device_now
    if _raw_stream is None:        # the handle and the number alone, where this torch gives them, spare a Stream object and a check per call
        t = _torch()
        _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (lambda device: t.cuda.current_stream(device).cuda_stream)
        _device_now = getattr(t._C, "_cuda_getDevice", None) or t.cuda.current_device
    now = _device_now()
    if now != device or (stream is not None and stream.device_index != now):
        raise ValueError(f"the current device is {now}, the tensors are on device {device}" + ("" if stream is None else f", the stream on {stream.device_index}"))
    return _raw_stream(now) if stream is None else stream.cuda_stream


def ivf_kv_append(step, cache, k, v, rotary=None, positions=None, q=None, q_out=None, interleaved=False, stream=None):
    """Appends the new tokens' k and v [tokens, heads, d] to the cache; with rotary [positions, rot] float32 (cosines,
    then sines) keys and q [tokens, query heads, d] are rotated.  Returns q_out (default: a new tensor)."""
    n, dev = step.n_tokens, cache.device
    if step.device != dev:
        raise ValueError(f"the step is on device {step.device}, the cache on {dev}")
    on = _on(stream, dev)
    kr, vr = _rows(k, n, cache.heads, cache, "k"), _rows(v, n, cache.heads, cache, "v")
    qr = qo = rp = pp = None
    hq = n_pos = rot = 0
    if q is not None:
        if q_out is None:
            q_out = _new(stream, q.shape, q.dtype)
        hq = q.shape[1]
        qr, qo = _rows(q, n, hq, cache, "q"), _rows(q_out, n, hq, cache, "q_out")
    elif q_out is not None:
        raise ValueError("q_out without q")
    if rotary is not None:
        if rotary.dtype is not _torch().float32 or rotary.get_device() != dev or not rotary.is_contiguous() or rotary.dim() != 2:
            raise ValueError("rotary must be a contiguous float32 tensor [positions, rot] on the cache's device")
        n_pos, rot = rotary.shape
        rp = rotary.data_ptr()
    if positions is not None:
        pp = _i32(positions, (n,), dev, "positions")
    status = load().ivf_kv_append(step.ref, cache.ref, kr, vr, rp, n_pos, rot, 1 if interleaved else 0, pp, qr, qo, hq, on)
    if status != 0:
        _check(status)
    return q_out


def ivf_attend(step, cache, q, out=None, lse=None, scale=None, window=0, sinks=0, workspace=None, stream=None):
    """Attention of the new tokens q [tokens, query heads, d] over the cache; returns out (default: a new tensor).
    lse: float32 [tokens, query heads] or None.  scale: default d ** -0.5.  workspace: a contiguous CUDA tensor of
    at least ivf_attend_workspace() bytes, default one for this call."""
    n, dev = step.n_tokens, cache.device
    if step.device != dev:
        raise ValueError(f"the step is on device {step.device}, the cache on {dev}")
    on = _on(stream, dev)
    if out is None:
        out = _new(stream, q.shape, q.dtype)
    hq = q.shape[1]
    qr, qo = _rows(q, n, hq, cache, "q"), _rows(out, n, hq, cache, "out")
    lp = wp = None
    wn = 0
    if lse is not None:
        if lse.dtype is not _torch().float32 or lse.get_device() != dev or not lse.is_contiguous() or lse.shape != (n, hq):
            raise ValueError("lse must be a contiguous float32 tensor [tokens, query heads] on the cache's device")
        lp = lse.data_ptr()
    if workspace is None:
        wn = ivf_attend_workspace(step, cache, hq, window, sinks)
        if wn:
            workspace = _workspace(wn, stream)
            wp = workspace.data_ptr()
    else:
        wp, wn = _room(workspace, dev)
    status = load().ivf_attend(step.ref, cache.ref, qr, hq, qo, lp, cache.d ** -0.5 if scale is None else scale, window, sinks, wp, wn, on)
    if status != 0:
        _check(status)
    return out


def ivf_attend_workspace(step, cache, n_q_heads, window=0, sinks=0):
    """Bytes of workspace of ivf_attend with these arguments."""
    key = (cache.heads, cache.d, cache.page, cache.pages, cache.quantised, n_q_heads, window, sinks)
    need = step._need.get(key)
    if need is None:
        n = C.c_size_t(0)
        _check(load().ivf_attend_workspace(step.ref, cache.ref, n_q_heads, window, sinks, C.byref(n)))
        need = step._need[key] = n.value
    return need


def ivf_kv_read(step, cache, out_off, k, v, first=None, stream=None):
    """Reads keys and values out of the cache into k and v [rows, heads, d] of its rows' type: rows out_off[s] .. out_off[s + 1]
    become the keys first[s] (default 0) and on of sequence s.  out_off [sequences + 1] and first [sequences] are int32 CUDA tensors.
    Returns k and v."""
    dev, n = cache.device, k.shape[0]
    if step.device != dev:
        raise ValueError(f"the step is on device {step.device}, the cache on {dev}")
    on = _on(stream, dev)
    kr, vr = _rows(k, n, cache.heads, cache, "k"), _rows(v, n, cache.heads, cache, "v")
    op = _i32(out_off, (step.arg.n_seq + 1,), dev, "out_off")
    fp = None if first is None else _i32(first, (step.arg.n_seq,), dev, "first")
    if n:
        _check(load().ivf_kv_read(step.ref, cache.ref, op, fp, n, kr, vr, on))
    return k, v


@functools.lru_cache(maxsize=64)             # a function of the sizes alone
def ivf_verify_workspace(n_seq, n_tokens, vocab):
    """Bytes of workspace of ivf_verify_draft with these sizes."""
    n = C.c_size_t(0)
    _check(load().ivf_verify_workspace(n_seq, n_tokens, vocab, C.byref(n)))
    return n.value


def _matrix(a, n_rows, what):
    """[n_rows, vocab] with the entries of a row side by side; the distance of its rows."""
    if a.dim() != 2 or a.shape[0] != n_rows or a.stride(1) != 1:
        raise ValueError(f"{what} must be [{n_rows}, vocab] with contiguous rows")
    return a.stride(0) if n_rows > 1 else a.shape[1]


def ivf_verify_draft(step, logits, tokens, uniform=None, draft=None, scale=1.0, lens_out=None, workspace=None, stream=None):
    """Verifies the drafted tokens of a step: of each sequence's new tokens (int32 [tokens]) the first is settled, the others are
    drafts.  logits [tokens, vocab] (float32, float16 or bfloat16) is what the target says behind each token, uniform float32 [tokens]
    in [0, 1) decides on the drafts and, by that of the settled token, on the token that follows.  draft: float32 [tokens, vocab], the
    probabilities that the drafts were drawn from, None where they were not drawn (copied text).  scale: the inverse of the temperature,
    0: the largest logit alone.  Returns per sequence the number of accepted drafts, the token that follows them, and the
    lengths less the refused ones (in lens_out, which may be the step's lens)."""
    t = _torch()
    dev, n = step.device, step.n_tokens
    on = _on(stream, dev)
    if logits.get_device() != dev:
        raise _elsewhere("logits", logits, dev)
    stride, vocab, dtype = _matrix(logits, n, "logits"), logits.shape[1], _code(logits.dtype)
    tp = _i32(tokens, (n,), dev, "tokens")
    up = dp = None
    by_draft = 0
    if uniform is not None:
        if uniform.dtype is not t.float32 or uniform.get_device() != dev or not uniform.is_contiguous() or uniform.shape != (n,):
            raise ValueError("uniform must be a contiguous float32 tensor [tokens] on the step's device")
        up = uniform.data_ptr()
    if draft is not None:
        if draft.dtype is not t.float32 or draft.get_device() != dev or draft.shape[-1] != vocab:
            raise ValueError("draft must be a float32 tensor [tokens, vocab] on the step's device")
        by_draft, dp = _matrix(draft, n, "draft"), draft.data_ptr()
    # what comes back is one allocation
    s = step.arg.n_seq
    out = _new(stream, (3 if lens_out is None else 2, s), t.int32)
    at = out.data_ptr()
    if lens_out is None:
        (accepted, follows, lens_out), lp = out.unbind(0), at + 8 * s
    else:
        (accepted, follows), lp = out.unbind(0), _i32(lens_out, (s,), dev, "lens_out")
    need = ivf_verify_workspace(s, n, vocab)
    if workspace is None:
        workspace = _workspace(need, stream)
        wp, wn = workspace.data_ptr(), need
    else:
        wp, wn = _room(workspace, dev)
    status = load().ivf_verify_draft(step.ref, logits.data_ptr(), stride, dtype, vocab, scale, tp, up, dp, by_draft, at, at + 4 * s, lp, wp, wn, on)
    if status != 0:
        _check(status)
    return accepted, follows, lens_out


@functools.lru_cache(maxsize=64)             # a function of the sizes alone
def ivf_beam_workspace(n_prompts, beams_in, vocab, beams_out):
    """Bytes of workspace of ivf_beam_step with these sizes."""
    n = C.c_size_t(0)
    _check(load().ivf_beam_workspace(n_prompts, beams_in, vocab, beams_out, C.byref(n)))
    return n.value


def _state(src, dst, rows_in, rows_out, device):
    """A state and its destination: rows of the same contiguous elements, evenly spaced."""
    if src.dtype is not dst.dtype or src.get_device() != device or dst.get_device() != device:
        raise ValueError("a state and its destination must be tensors of the same type on the logits' device")
    before, after = src.shape, dst.shape
    if before[0] != rows_in or after[0] != rows_out or before[1:] != after[1:]:
        raise ValueError("a state has a row per beam, before and after")
    if not (src.is_contiguous() or src[0].is_contiguous()) or not (dst.is_contiguous() or dst[0].is_contiguous()):
        raise ValueError("the rows of a state must be contiguous")
    size = src.itemsize
    row = src.numel() // rows_in * size
    return BeamStateArg(src.data_ptr(), dst.data_ptr(), row, src.stride(0) * size if rows_in > 1 else row, dst.stride(0) * size if rows_out > 1 else row)


def ivf_beam_step(logits, scores, beams_out=None, done=None, eos=-1, states=(), workspace=None, stream=None):
    """One step of a beam search.  logits [prompts, beams, vocab] (float32, float16 or bfloat16, rows evenly spaced),
    scores [prompts, beams] float32, done [prompts, beams] bool or uint8, or None.  states: pairs (from, to) of
    CUDA tensors with a row per beam, before and after (prompts * beams and prompts * beams_out rows, each row
    contiguous).  Returns scores, parents (row of logits), tokens and done, each [prompts, beams_out]."""
    t = _torch()
    dev = logits.get_device()
    if logits.dim() != 3 or dev < 0 or logits.stride(2) != 1:
        raise ValueError("logits must be a CUDA tensor [prompts, beams, vocab] with contiguous rows")
    on = _on(stream, dev)
    p, b, vocab = logits.shape
    by_prompt, stride, _ = logits.stride()
    if b == 1:
        stride = by_prompt if p > 1 else vocab
    elif p > 1 and by_prompt != b * stride:
        raise ValueError("the rows of logits must be evenly spaced")
    if scores.dtype is not t.float32 or scores.get_device() != dev or not scores.is_contiguous() or scores.shape != (p, b):
        raise ValueError("scores must be a contiguous float32 tensor [prompts, beams] on the logits' device")
    dp = None
    if done is not None:
        if done.dtype not in (t.bool, t.uint8) or done.get_device() != dev or not done.is_contiguous() or done.shape != (p, b):
            raise ValueError("done must be a contiguous bool or uint8 tensor [prompts, beams] on the logits' device")
        dp = done.data_ptr()
    n = b if beams_out is None else beams_out
    args = (BeamStateArg * len(states))(*[_state(src, dst, p * b, p * n, dev) for src, dst in states]) if states else None
    need = ivf_beam_workspace(p, b, vocab, n)
    # the scores, parents and tokens are one allocation
    out = _new(stream, (3, p, n), t.int32)
    score, parent, token = out.unbind(0)
    score = score.view(t.float32)
    fin = _new(stream, (p, n), t.bool)
    if workspace is None:
        workspace = _workspace(need, stream)
        wp, wn = workspace.data_ptr(), need
    else:
        wp, wn = _room(workspace, dev)
    at = out.data_ptr()
    status = load().ivf_beam_step(logits.data_ptr(), stride, _code(logits.dtype), p, b, vocab, scores.data_ptr(), dp, eos, n,
                                  at, at + 4 * p * n, at + 8 * p * n, fin.data_ptr(), args, len(states),
                                  wp, wn, on)
    if status != 0:
        _check(status)
    return score, parent, token, fin
