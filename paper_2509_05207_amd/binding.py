"""ctypes binding of librapidgnn_hip.so: same names as include/rapidgnn.h.

Argument marshalling only.  Every step of the data path runs in the library's
HIP kernels; torch is used for device memory (inputs, the gather output) and
for stream handles.  There is no CPU fallback: if the library has not been
built, importing the entry points raises.
"""
import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "librapidgnn_hip.so")

RG_OK, RG_EINVAL, RG_ENOMEM, RG_EHIP, RG_ERANGE, RG_EIO = 0, -1, -2, -3, -4, -5
RG_MAX_HOPS, RG_MAX_FANOUT, RG_MAX_BATCHES = 8, 1984, 65535
KERNEL_GROUPS = ("sampler", "frontier", "shuffle_sort", "histogram", "topk", "plan", "cache_fill", "gather", "gather_miss", "sample_offsets", "blocks")

EXPORTS = ("rg_last_error", "rg_graph_validate", "rg_build_schedule", "rg_schedule_info", "rg_schedule_frontier",
           "rg_schedule_samples", "rg_build_cache", "rg_cache_view", "rg_gather_batch", "rg_schedule_destroy",
           "rg_cache_destroy", "rg_trim_memory", "rg_profile_enable", "rg_profile_reset", "rg_profile_read",
           "rg_cache_pair_create", "rg_cache_pair_begin_next", "rg_cache_pair_swap", "rg_cache_pair_primary",
           "rg_cache_pair_table_bytes", "rg_cache_pair_destroy",
           "rg_prefetcher_create", "rg_prefetcher_fill", "rg_prefetcher_acquire", "rg_prefetcher_release",
           "rg_prefetcher_depth", "rg_prefetcher_destroy", "rg_schedule_build_blocks", "rg_schedule_block",
           "rg_classify_batch", "rg_build_schedule_with", "rg_gather_batches",
           "rg_schedule_save", "rg_schedule_load", "rg_gather_batch_noalloc", "rg_schedule_seeds", "rg_schedule_load_range",
           "rg_layer_norm", "rg_layer_norm_workspace", "rg_layer_norm_backward",
           "rg_update_workspace", "rg_orthogonalize", "rg_muon_step",
           "rg_rows8_bytes", "rg_quantize_rows", "rg_dequantize_rows", "rg_rows8_product_workspace", "rg_rows8_product",
           "rg_rows8_product_backward_workspace", "rg_rows8_product_backward")


class RgError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"rapidgnn status {status}: {message}")
        self.status = status


class rg_graph(C.Structure):
    _fields_ = [("n_nodes", C.c_int64), ("indptr", C.c_void_p), ("indices", C.c_void_p)]


class rg_features(C.Structure):
    _fields_ = [("is_local", C.c_void_p), ("row_of", C.c_void_p), ("local_rows", C.c_void_p), ("local_stride", C.c_uint64),
                ("remote_rows", C.c_void_p), ("remote_stride", C.c_uint64), ("row_bytes", C.c_uint32)]


class rg_gather_stats(C.Structure):
    _fields_ = [("n_rows", C.c_uint64), ("n_local", C.c_uint64), ("n_hit", C.c_uint64), ("n_miss", C.c_uint64)]


class rg_update(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("grad_stride", C.c_uint64), ("weight", C.c_void_p), ("weight_stride", C.c_uint64),
                ("momentum", C.c_void_p), ("momentum_stride", C.c_uint64), ("momentum_out", C.c_void_p), ("momentum_out_stride", C.c_uint64),
                ("out", C.c_void_p), ("out_stride", C.c_uint64), ("rows", C.c_uint32), ("cols", C.c_uint32)]


ALLOC_FN = C.CFUNCTYPE(C.c_void_p, C.c_uint64, C.c_int, C.c_void_p)
FREE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_int, C.c_void_p)


class rg_allocator(C.Structure):
    _fields_ = [("alloc", ALLOC_FN), ("free", FREE_FN), ("ctx", C.c_void_p)]


_lib = None


def use_library(path):
    """Load another build of the same library (the profiling build with phase timers) instead of the default one.
    Must be called before the first call of lib()."""
    global _LIB_PATH
    if _lib is not None:
        raise RuntimeError("the library is already loaded")
    _LIB_PATH = os.path.abspath(path)


def lib():
    """The loaded library; raises if it has not been built (python -m paper_2509_05207_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2509_05207_amd.build` "
                               "(there is no fallback path)")
        L = C.CDLL(_LIB_PATH)
        vp, u64, u32, i64 = C.c_void_p, C.c_uint64, C.c_uint32, C.c_int64
        P = C.POINTER
        L.rg_last_error.restype = C.c_char_p
        L.rg_graph_validate.argtypes = [P(rg_graph), vp, P(u64)]
        L.rg_build_schedule.argtypes = [P(rg_graph), vp, u64, u32, P(u32), u32, u64, u32, u32, P(rg_allocator), vp, P(vp)]
        L.rg_build_schedule_with.argtypes = [P(rg_graph), vp, u64, u32, P(u32), u32, u64, u32, u32, u32, P(rg_allocator), vp, P(vp)]
        L.rg_schedule_info.argtypes = [vp, P(u32), P(u32), P(i64)]
        L.rg_schedule_frontier.argtypes = [vp, u32, P(vp), P(vp), P(vp)]
        L.rg_schedule_samples.argtypes = [vp, u32, P(vp), P(vp), P(i64)]
        L.rg_schedule_seeds.argtypes = [vp, P(vp), P(vp)]
        L.rg_build_cache.argtypes = [P(vp), u32, P(rg_features), u64, P(rg_allocator), vp, P(vp)]
        L.rg_cache_view.argtypes = [vp, P(u64), P(vp), P(vp), P(vp), P(vp), P(u64)]
        L.rg_gather_batch.argtypes = [vp, vp, P(rg_features), u32, vp, u64, u64, vp, vp, P(rg_gather_stats)]
        L.rg_gather_batch_noalloc.argtypes = [vp, vp, P(rg_features), u32, vp, u64, u64, vp, P(rg_gather_stats)]
        L.rg_schedule_destroy.argtypes = [vp]; L.rg_schedule_destroy.restype = None
        L.rg_cache_destroy.argtypes = [vp]; L.rg_cache_destroy.restype = None
        L.rg_trim_memory.argtypes = []; L.rg_trim_memory.restype = None
        L.rg_profile_enable.argtypes = [C.c_int]; L.rg_profile_enable.restype = None
        L.rg_profile_reset.argtypes = []; L.rg_profile_reset.restype = None
        L.rg_profile_read.argtypes = [P(C.c_double), P(u64)]
        L.rg_schedule_save.argtypes = [vp, C.c_char_p, vp]
        L.rg_schedule_load.argtypes = [C.c_char_p, P(rg_allocator), vp, P(vp)]
        L.rg_schedule_load_range.argtypes = [C.c_char_p, u32, u32, P(rg_allocator), vp, P(vp)]
        L.rg_gather_batches.argtypes = [vp, vp, P(rg_features), u32, u32, vp, u64, u64, vp, vp, P(rg_gather_stats)]
        L.rg_classify_batch.argtypes = [vp, vp, P(rg_features), u32, vp, P(rg_gather_stats)]
        L.rg_schedule_build_blocks.argtypes = [vp, u64, vp]
        L.rg_schedule_block.argtypes = [vp, u32, P(vp)]
        L.rg_cache_pair_create.argtypes = [vp, P(rg_features), u64, P(rg_allocator), vp, P(vp)]
        L.rg_cache_pair_begin_next.argtypes = [vp, vp]
        L.rg_cache_pair_swap.argtypes = [vp, C.c_int, P(C.c_int)]
        L.rg_cache_pair_primary.argtypes = [vp]; L.rg_cache_pair_primary.restype = vp
        L.rg_cache_pair_table_bytes.argtypes = [vp]; L.rg_cache_pair_table_bytes.restype = u64
        L.rg_cache_pair_destroy.argtypes = [vp]; L.rg_cache_pair_destroy.restype = None
        L.rg_prefetcher_create.argtypes = [vp, vp, P(rg_features), u32, P(vp), u64, u64, P(vp)]
        L.rg_prefetcher_fill.argtypes = [vp, P(u32)]
        L.rg_prefetcher_acquire.argtypes = [vp, vp, P(u32), P(vp), P(rg_gather_stats), P(C.c_int)]
        L.rg_prefetcher_release.argtypes = [vp, vp]
        L.rg_prefetcher_depth.argtypes = [vp, P(u32), P(u32)]
        L.rg_prefetcher_destroy.argtypes = [vp]; L.rg_prefetcher_destroy.restype = None
        L.rg_layer_norm.argtypes = [vp, u64, u64, u64, u32, vp, vp, u32, C.c_float, vp, u64, vp, vp, vp]
        L.rg_layer_norm_workspace.argtypes = [u64, u64, u32, P(u64)]
        L.rg_layer_norm_backward.argtypes = [vp, u64, vp, u64, u64, u64, u32, vp, u32, vp, vp, vp, u64, vp, vp, vp, u64, vp]
        L.rg_update_workspace.argtypes = [P(rg_update), u32, u32, P(u64)]
        L.rg_orthogonalize.argtypes = [P(rg_update), u32, u32, u32, C.c_float, vp, u64, vp]
        L.rg_muon_step.argtypes = [P(rg_update), u32, u32, C.c_float, C.c_float, C.c_float, C.c_int, u32, C.c_float, vp, u64, vp]
        L.rg_rows8_bytes.argtypes = [u64, P(u64)]
        L.rg_quantize_rows.argtypes = [vp, u64, u64, u64, u32, vp, u64, vp, u64, vp]
        L.rg_dequantize_rows.argtypes = [vp, u64, u64, u64, vp, u64, u32, vp, u64, vp]
        L.rg_rows8_product_workspace.argtypes = [u64, u64, u64, u32, P(u64)]
        L.rg_rows8_product.argtypes = [vp, u64, u64, vp, u64, u64, u64, vp, u32, vp, u64, u32, vp, u64, vp]
        L.rg_rows8_product_backward_workspace.argtypes = [u64, u64, u64, u32, C.c_int, C.c_int, C.c_int, P(u64)]
        L.rg_rows8_product_backward.argtypes = [vp, u64, vp, u64, vp, u64, u64, u64, u64, u32, vp, u64, vp, u64, vp, u32, vp, u64, vp]
        for name in ("rg_rows8_bytes", "rg_quantize_rows", "rg_dequantize_rows", "rg_rows8_product_workspace", "rg_rows8_product",
                     "rg_rows8_product_backward_workspace", "rg_rows8_product_backward"):
            getattr(L, name).restype = C.c_int32
        for name in ("rg_layer_norm", "rg_layer_norm_workspace", "rg_layer_norm_backward", "rg_update_workspace", "rg_orthogonalize", "rg_muon_step"):
            getattr(L, name).restype = C.c_int32
        for name in ("rg_graph_validate", "rg_build_schedule", "rg_schedule_info", "rg_schedule_frontier", "rg_schedule_samples",
                     "rg_build_cache", "rg_cache_view", "rg_gather_batch", "rg_profile_read",
                     "rg_cache_pair_create", "rg_cache_pair_begin_next", "rg_cache_pair_swap",
                     "rg_prefetcher_create", "rg_prefetcher_fill", "rg_prefetcher_acquire", "rg_prefetcher_release",
                     "rg_prefetcher_depth", "rg_schedule_build_blocks", "rg_schedule_block",
           "rg_classify_batch", "rg_build_schedule_with", "rg_gather_batches",
           "rg_schedule_save", "rg_schedule_load", "rg_gather_batch_noalloc", "rg_schedule_seeds", "rg_schedule_load_range"):
            getattr(L, name).restype = C.c_int32
        _lib = L
    return _lib


def _check(status):
    if status != RG_OK:
        raise RgError(status, lib().rg_last_error().decode())


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _dev_ptr(t, dtype=None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "expected a contiguous device tensor"
    if dtype is not None:
        assert t.dtype == dtype, f"expected {dtype}, got {t.dtype}"
    return C.c_void_p(t.data_ptr())


class _DevView:
    """Zero-copy view of library-owned device memory for torch.as_tensor."""

    def __init__(self, ptr, n, typestr):
        self.__cuda_array_interface__ = {"shape": (int(n),), "typestr": typestr, "data": (int(ptr), False), "version": 2}


def _view(ptr, n, typestr, owner):
    if n == 0 or not ptr:
        dt = {"<i4": torch.int32, "<i8": torch.int64, "<u1": torch.uint8}[typestr]
        return torch.empty(0, dtype=dt, device="cuda")
    t = torch.as_tensor(_DevView(ptr, n, typestr), device="cuda")
    t._rg_owner = owner          # keep the handle alive as long as the view
    return t


def _graph_struct(indptr, indices):
    n = indptr.numel() - 1
    return rg_graph(n, _dev_ptr(indptr, torch.int64), _dev_ptr(indices, torch.int32) if indices.numel() else None)


def rg_graph_validate(indptr, indices, stream=None):
    """Number of violations of the CSR precondition (0 = valid)."""
    g = _graph_struct(indptr, indices)
    bad = C.c_uint64(0)
    _check(lib().rg_graph_validate(C.byref(g), _stream_ptr(stream), C.byref(bad)))
    return bad.value


class Schedule:
    def __init__(self, handle, keep=None):
        self.h = C.c_void_p(handle)
        self._keep = keep            # the allocator the handle's memory came from must outlive the handle
        nb, L, nn = C.c_uint32(), C.c_uint32(), C.c_int64()
        _check(lib().rg_schedule_info(self.h, C.byref(nb), C.byref(L), C.byref(nn)))
        self.n_batches, self.L, self.n_nodes = nb.value, L.value, nn.value

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rg_schedule_destroy(self.h)
            self.h = None


class Cache:
    def __init__(self, handle, keep):
        self.h = C.c_void_p(handle)
        self._keep = keep            # borrowed inputs (feature tensors, schedules) must outlive the cache

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rg_cache_destroy(self.h)
            self.h = None


RG_SAMPLER_KEYS, RG_SAMPLER_POSITIONS = 0, 1


def rg_build_schedule(indptr, indices, train_nodes, batch_size, fanout, s0=0, worker=0, epoch=0, allocator=None, stream=None):
    g = _graph_struct(indptr, indices)
    fan = (C.c_uint32 * max(len(fanout), 1))(*[int(x) for x in fanout])
    out = C.c_void_p()
    T = train_nodes.numel()
    _check(lib().rg_build_schedule(C.byref(g), _dev_ptr(train_nodes, torch.int32) if T else None, T, int(batch_size), fan,
                                   len(fanout), int(s0), int(worker), int(epoch),
                                   C.byref(allocator) if allocator is not None else None, _stream_ptr(stream), C.byref(out)))
    return Schedule(out.value, allocator)


def rg_build_schedule_with(indptr, indices, train_nodes, batch_size, fanout, s0=0, worker=0, epoch=0, sampler=RG_SAMPLER_KEYS,
                           allocator=None, stream=None):
    g = _graph_struct(indptr, indices)
    fan = (C.c_uint32 * max(len(fanout), 1))(*[int(x) for x in fanout])
    out = C.c_void_p()
    T = train_nodes.numel()
    _check(lib().rg_build_schedule_with(C.byref(g), _dev_ptr(train_nodes, torch.int32) if T else None, T, int(batch_size), fan,
                                        len(fanout), int(s0), int(worker), int(epoch), int(sampler),
                                        C.byref(allocator) if allocator is not None else None, _stream_ptr(stream), C.byref(out)))
    return Schedule(out.value, allocator)


def rg_schedule_save(s, path, stream=None):
    _check(lib().rg_schedule_save(s.h, os.fsencode(path), _stream_ptr(stream)))


def rg_schedule_load(path, allocator=None, stream=None):
    out = C.c_void_p()
    _check(lib().rg_schedule_load(os.fsencode(path), C.byref(allocator) if allocator is not None else None, _stream_ptr(stream),
                                  C.byref(out)))
    return Schedule(out.value, allocator)


def rg_schedule_load_range(path, first_batch, n_batches, allocator=None, stream=None):
    """Batches [first_batch, first_batch + n_batches) of a schedule file as a schedule of their own."""
    out = C.c_void_p()
    _check(lib().rg_schedule_load_range(os.fsencode(path), int(first_batch), int(n_batches),
                                        C.byref(allocator) if allocator is not None else None, _stream_ptr(stream), C.byref(out)))
    return Schedule(out.value, allocator)


def rg_schedule_frontier(s, hop):
    """(ids device tensor, batch offsets device tensor, batch offsets numpy)."""
    ids, offd, offh = C.c_void_p(), C.c_void_p(), C.c_void_p()
    _check(lib().rg_schedule_frontier(s.h, int(hop), C.byref(ids), C.byref(offd), C.byref(offh)))
    off_host = np.ctypeslib.as_array(C.cast(offh, C.POINTER(C.c_int64)), shape=(s.n_batches + 1,)).copy()
    n = int(off_host[-1])
    return _view(ids.value, n, "<i4", s), _view(offd.value, s.n_batches + 1, "<i8", s), off_host


def rg_schedule_seeds(s):
    """(seeds device tensor: the shuffled train nodes; batch offsets device tensor [n_batches + 1])."""
    ids, offd = C.c_void_p(), C.c_void_p()
    _check(lib().rg_schedule_seeds(s.h, C.byref(ids), C.byref(offd)))
    off = _view(offd.value, s.n_batches + 1, "<i8", s)
    return _view(ids.value, int(off[-1].item()) if s.n_batches else 0, "<i4", s), off


def rg_schedule_samples(s, hop):
    """(samp_off device tensor [|U_hop| + 1], samp_nbr device tensor)."""
    so, sn, ns = C.c_void_p(), C.c_void_p(), C.c_int64()
    _check(lib().rg_schedule_samples(s.h, int(hop), C.byref(so), C.byref(sn), C.byref(ns)))
    _, _, off_host = rg_schedule_frontier(s, hop)
    return _view(so.value, int(off_host[-1]) + 1, "<i8", s), _view(sn.value, ns.value, "<i4", s)


def rg_schedule_build_blocks(s, workspace_limit_bytes=0, stream=None):
    _check(lib().rg_schedule_build_blocks(s.h, int(workspace_limit_bytes), _stream_ptr(stream)))


def rg_schedule_block(s, hop):
    """src_pos device tensor: block-local source index of every sample of the hop."""
    p, ns = C.c_void_p(), C.c_int64()
    _check(lib().rg_schedule_block(s.h, int(hop), C.byref(p)))
    _check(lib().rg_schedule_samples(s.h, int(hop), None, None, C.byref(ns)))
    return _view(p.value, ns.value, "<i4", s)


def make_features(is_local, row_of, local_rows, remote_rows, row_bytes, local_stride=None, remote_stride=None):
    """rg_features over torch tensors.  remote_rows may be a device tensor or a pinned host tensor."""
    assert remote_rows.is_cuda or remote_rows.is_pinned() or remote_rows.numel() == 0, "remote rows must be device-visible"
    assert local_rows.is_contiguous() and remote_rows.is_contiguous()
    ls = local_stride if local_stride is not None else (local_rows.stride(0) * local_rows.element_size() if local_rows.dim() == 2 else row_bytes)
    rs = remote_stride if remote_stride is not None else (remote_rows.stride(0) * remote_rows.element_size() if remote_rows.dim() == 2 else row_bytes)
    f = rg_features(_dev_ptr(is_local, torch.uint8), _dev_ptr(row_of, torch.int32), C.c_void_p(local_rows.data_ptr()), int(ls),
                    C.c_void_p(remote_rows.data_ptr()), int(rs), int(row_bytes))
    f._keep = (is_local, row_of, local_rows, remote_rows)
    return f


def rg_build_cache(schedules, features, K, allocator=None, stream=None):
    hs = (C.c_void_p * len(schedules))(*[s.h for s in schedules])
    out = C.c_void_p()
    _check(lib().rg_build_cache(hs, len(schedules), C.byref(features), int(K),
                                C.byref(allocator) if allocator is not None else None, _stream_ptr(stream), C.byref(out)))
    return Cache(out.value, (features, list(schedules), allocator))


class CacheView(dict):
    """K_eff, cache_ids, rows (device tensors over the cache's memory) and stride, fetched at once; "freq" and
    "slot_of" are fetched when first read, since the library may have to make those two arrays (4 bytes per node
    each) for the occasion."""

    def __init__(self, c, n_nodes):
        super().__init__()
        self._c, self._n = c, n_nodes
        k, ids, rows, stride = C.c_uint64(), C.c_void_p(), C.c_void_p(), C.c_uint64()
        _check(lib().rg_cache_view(c.h, C.byref(k), C.byref(ids), None, None, C.byref(rows), C.byref(stride)))
        self.update(K_eff=k.value, cache_ids=_view(ids.value, k.value, "<i4", c),
                    rows=_view(rows.value, k.value * stride.value, "<u1", c), stride=stride.value)

    def __missing__(self, key):
        p = C.c_void_p()
        if key == "freq":
            _check(lib().rg_cache_view(self._c.h, None, None, C.byref(p), None, None, None))
        elif key == "slot_of":
            _check(lib().rg_cache_view(self._c.h, None, None, None, C.byref(p), None, None))
        else:
            raise KeyError(key)
        self[key] = _view(p.value, self._n, "<i4", self._c)      # counts are < 2^31: reading them as int32 is exact
        return self[key]


def rg_cache_view(c, n_nodes):
    """Mapping with K_eff, cache_ids, freq, slot_of, rows (device tensors) and stride; see CacheView."""
    return CacheView(c, n_nodes)


def rg_gather_batch(s, c, features, batch, out, out_stride=None, out_capacity_rows=None, stream=None, side_stream=None,
                    want_stats=True):
    """Fills `out` (device tensor) with the batch's feature rows; returns the stats dict."""
    assert out.is_cuda and out.is_contiguous()
    if out_stride is None:
        out_stride = out.stride(0) * out.element_size()
    if out_capacity_rows is None:
        out_capacity_rows = out.numel() * out.element_size() // out_stride
    st = rg_gather_stats()
    side = _stream_ptr(side_stream) if side_stream is not None else None
    _check(lib().rg_gather_batch(s.h, c.h if c is not None else None, C.byref(features), int(batch), C.c_void_p(out.data_ptr()),
                                 int(out_stride), int(out_capacity_rows), _stream_ptr(stream), side,
                                 C.byref(st) if want_stats else None))
    return dict(n_rows=st.n_rows, n_local=st.n_local, n_hit=st.n_hit, n_miss=st.n_miss) if want_stats else None


RG_NOALLOC_MAX_ROWS = 1 << 22


def rg_gather_batch_noalloc(s, c, features, batch, out, out_stride=None, out_capacity_rows=None, stream=None, want_stats=True):
    """rg_gather_batch through the entry point that allocates nothing; returns the stats dict (None without stats)."""
    assert out.is_cuda and out.is_contiguous()
    if out_stride is None:
        out_stride = out.stride(0) * out.element_size()
    if out_capacity_rows is None:
        out_capacity_rows = out.numel() * out.element_size() // out_stride
    st = rg_gather_stats()
    _check(lib().rg_gather_batch_noalloc(s.h, c.h if c is not None else None, C.byref(features), int(batch), C.c_void_p(out.data_ptr()),
                                         int(out_stride), int(out_capacity_rows), _stream_ptr(stream), C.byref(st) if want_stats else None))
    return dict(n_rows=st.n_rows, n_local=st.n_local, n_hit=st.n_hit, n_miss=st.n_miss) if want_stats else None


def rg_gather_batches(s, c, features, first_batch, n_batches, out, out_stride=None, out_capacity_rows=None, stream=None,
                      side_stream=None, want_stats=True):
    """Blocks of batches [first_batch, first_batch + n_batches) back to back in `out`; returns the list of stats dicts."""
    assert out.is_cuda and out.is_contiguous()
    if out_stride is None:
        out_stride = out.stride(0) * out.element_size()
    if out_capacity_rows is None:
        out_capacity_rows = out.numel() * out.element_size() // out_stride
    st = (rg_gather_stats * max(int(n_batches), 1))()
    side = _stream_ptr(side_stream) if side_stream is not None else None
    _check(lib().rg_gather_batches(s.h, c.h if c is not None else None, C.byref(features), int(first_batch), int(n_batches),
                                   C.c_void_p(out.data_ptr()), int(out_stride), int(out_capacity_rows), _stream_ptr(stream), side,
                                   st if want_stats else None))
    if not want_stats:
        return None
    return [dict(n_rows=x.n_rows, n_local=x.n_local, n_hit=x.n_hit, n_miss=x.n_miss) for x in st[:int(n_batches)]]


def rg_classify_batch(s, c, features, batch, stream=None):
    """The batch's counts (rows, local, hits, misses) without gathering."""
    st = rg_gather_stats()
    _check(lib().rg_classify_batch(s.h, c.h if c is not None else None, C.byref(features), int(batch), _stream_ptr(stream), C.byref(st)))
    return dict(n_rows=st.n_rows, n_local=st.n_local, n_hit=st.n_hit, n_miss=st.n_miss)


class _BorrowedCache:
    """A cache handle owned by something else (a cache pair)."""

    def __init__(self, handle, owner):
        self.h = C.c_void_p(handle)
        self._owner = owner


class CachePair:
    def __init__(self, handle, keep):
        self.h = C.c_void_p(handle)
        self._keep = list(keep)

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rg_cache_pair_destroy(self.h)
            self.h = None


def rg_cache_pair_create(first_epoch, features, K, allocator=None, stream=None):
    out = C.c_void_p()
    _check(lib().rg_cache_pair_create(first_epoch.h, C.byref(features), int(K),
                                      C.byref(allocator) if allocator is not None else None, _stream_ptr(stream), C.byref(out)))
    return CachePair(out.value, (features, first_epoch, allocator))


def rg_cache_pair_begin_next(p, next_epoch):
    p._keep.append(next_epoch)
    _check(lib().rg_cache_pair_begin_next(p.h, next_epoch.h))


def rg_cache_pair_swap(p, wait=False):
    """True if C_sec was swapped in."""
    sw = C.c_int(0)
    _check(lib().rg_cache_pair_swap(p.h, 1 if wait else 0, C.byref(sw)))
    return bool(sw.value)


def rg_cache_pair_primary(p):
    return _BorrowedCache(lib().rg_cache_pair_primary(p.h), p)


def rg_cache_pair_table_bytes(p):
    return int(lib().rg_cache_pair_table_bytes(p.h))


class Prefetcher:
    def __init__(self, handle, keep, slots, out_stride):
        self.h = C.c_void_p(handle)
        self._keep = keep
        self.slots = slots
        self.out_stride = out_stride
        self._by_ptr = {t.data_ptr(): i for i, t in enumerate(slots)}

    def __del__(self):
        if getattr(self, "h", None) and _lib is not None:
            _lib.rg_prefetcher_destroy(self.h)
            self.h = None


def rg_prefetcher_create(s, c, features, slots, out_stride=None, slot_capacity_rows=None):
    """`slots`: list of Q equally sized contiguous device tensors, one staged feature block each."""
    Q = len(slots)
    assert all(t.is_cuda and t.is_contiguous() for t in slots)
    if out_stride is None:
        out_stride = slots[0].stride(0) * slots[0].element_size()
    if slot_capacity_rows is None:
        slot_capacity_rows = min(t.numel() * t.element_size() for t in slots) // out_stride
    ptrs = (C.c_void_p * max(Q, 1))(*[t.data_ptr() for t in slots])
    out = C.c_void_p()
    _check(lib().rg_prefetcher_create(s.h, c.h if c is not None else None, C.byref(features), Q, ptrs, int(out_stride),
                                      int(slot_capacity_rows), C.byref(out)))
    return Prefetcher(out.value, (s, c, features), list(slots), int(out_stride))


def rg_prefetcher_fill(p):
    n = C.c_uint32(0)
    _check(lib().rg_prefetcher_fill(p.h, C.byref(n)))
    return n.value


def rg_prefetcher_acquire(p, stream=None):
    """(batch, slot tensor, stats dict, was_staged) of the next batch in schedule order."""
    b, out, st, staged = C.c_uint32(), C.c_void_p(), rg_gather_stats(), C.c_int(0)
    _check(lib().rg_prefetcher_acquire(p.h, _stream_ptr(stream), C.byref(b), C.byref(out), C.byref(st), C.byref(staged)))
    stats = dict(n_rows=st.n_rows, n_local=st.n_local, n_hit=st.n_hit, n_miss=st.n_miss)
    return b.value, p.slots[p._by_ptr[out.value]], stats, bool(staged.value)


def rg_prefetcher_release(p, stream=None):
    _check(lib().rg_prefetcher_release(p.h, _stream_ptr(stream)))


def rg_prefetcher_depth(p):
    """(staged and not yet acquired, held by the consumer)."""
    a, h = C.c_uint32(), C.c_uint32()
    _check(lib().rg_prefetcher_depth(p.h, C.byref(a), C.byref(h)))
    return a.value, h.value


# ---------------------------------------------------------------- operators of the training step behind the gathered blocks
RG_F32, RG_BF16, RG_F16 = 0, 1, 2
_ELEMENT = {torch.float32: RG_F32, torch.bfloat16: RG_BF16, torch.float16: RG_F16}


def _rows(name, t, device, shape=None, dtype=None):
    """(address, stride in bytes) of a matrix on `device` (any GPU, if None) whose rows are contiguous."""
    assert t.dim() == 2 and (t.is_cuda if device is None else t.device == device), f"{name}: expected a matrix on {device or 'the device'}"
    assert shape is None or t.shape == shape, f"{name}: expected the shape {tuple(shape)}, got {tuple(t.shape)}"
    assert (dtype is None and t.dtype in _ELEMENT) or t.dtype == dtype, f"{name}: got {t.dtype}"
    along, across = t.stride()
    assert across == 1 or t.shape[1] <= 1, f"{name}: the elements of a row have to be contiguous"
    return t.data_ptr(), along * t.element_size()


def _vector(name, t, device, n, dtype):
    if t is None:
        return None
    assert t.device == device and t.dtype == dtype and t.shape == (n,) and t.is_contiguous(), f"{name}: expected {n} contiguous {dtype} on {device}"
    return t.data_ptr()


def _scratch(t, device):
    """(address, bytes) of a workspace."""
    assert t.device == device and t.is_contiguous(), f"workspace: expected a contiguous tensor on {device}"
    return t.data_ptr(), t.numel() * t.element_size()


def _written(*tensors):
    """Tells autograd that what lies in these was written over (a call writes through raw addresses, which it does not see)."""
    torch.autograd.graph.increment_version(tensors)


def _call(device, entry, *args):
    """The entry point with the operands' device the current one, to which the library's launches and questions go."""
    if device.index == torch._C._cuda_getDevice():
        _check(entry(*args))
    else:
        with torch.cuda.device(device):
            _check(entry(*args))


def _stream_and_use(device, stream, *made):
    """The raw handle of `stream`, the current one if None (what torch's own generated code asks for: a Stream object costs 3 us a call).  Tensors
    made here on the current stream are handed to work on a stream that is not."""
    current = torch._C._cuda_getCurrentRawStream(device.index)
    if stream is None:
        return current
    raw = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if raw != current:
        stream = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(raw)
        stream.wait_stream(torch.cuda.current_stream(device))        # what had their memory before may still be queued there
        for t in made:
            if t is not None:
                t.record_stream(stream)
    return raw


def rg_layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """(y, mean, rstd) of the rows of `x` (device matrix; rows may be padded).  out: where y goes (x itself: in place)."""
    shape, dt, device = x.shape, x.dtype, x.device
    xp, xs = _rows("x", x, None)
    n, d = shape
    y = x.new_empty(shape) if out is None else out
    yp, ys = (y.data_ptr(), d * y.element_size()) if out is None else _rows("out", y, device, shape, dt)
    wt = (weight if weight is not None else bias if bias is not None else x).dtype
    stats = torch.empty((2, n), dtype=torch.float32, device=device)
    sp = stats.data_ptr()
    st = _stream_and_use(device, stream, y if out is None else None, stats)
    _call(device, lib().rg_layer_norm, xp, xs, n, d, _ELEMENT[dt], _vector("weight", weight, device, d, wt), _vector("bias", bias, device, d, wt), _ELEMENT[wt],
          eps, yp, ys, sp, sp + 4 * n, st)
    if out is not None:
        _written(out)
    return y, stats[0], stats[1]


def rg_layer_norm_workspace(n_rows, n_cols, dtype):
    """Bytes of scratch that the backward pass takes."""
    b = C.c_uint64()
    _check(lib().rg_layer_norm_workspace(int(n_rows), int(n_cols), _ELEMENT[dtype], C.byref(b)))
    return b.value


def rg_layer_norm_backward(dy, x, weight, mean, rstd, want_dx=True, want_dweight=True, want_dbias=True, out=None, workspace=None, stream=None):
    """(dx, dweight, dbias); None for what is not wanted.  weight None: all ones (the gradients of weight and bias are then fp32).
    out: where dx goes (dy or x itself: in place); workspace: a device tensor of rg_layer_norm_workspace bytes, made here if None."""
    shape, dt, device = x.shape, x.dtype, x.device
    xp, xs = _rows("x", x, None)
    gp, gs = _rows("dy", dy, device, shape, dt)
    n, d = shape
    wt = weight.dtype if weight is not None else torch.float32
    dx, op, os_ = None, None, 0
    if want_dx:
        dx = x.new_empty(shape) if out is None else out
        op, os_ = _rows("out", dx, device, shape, dt)
    dw = torch.empty(d, dtype=wt, device=device) if want_dweight else None
    db = torch.empty(d, dtype=wt, device=device) if want_dbias else None
    made = workspace is None and (want_dweight or want_dbias)
    if made:
        b = C.c_uint64()
        _call(device, lib().rg_layer_norm_workspace, n, d, _ELEMENT[dt], C.byref(b))
        workspace = torch.empty(max(b.value, 1), dtype=torch.uint8, device=device)
    st = _stream_and_use(device, stream, dx if out is None else None, dw, db, workspace if made else None)
    wp, wb = (None, 0) if workspace is None else _scratch(workspace, device)
    _call(device, lib().rg_layer_norm_backward, gp, gs, xp, xs, n, d, _ELEMENT[dt], _vector("weight", weight, device, d, wt), _ELEMENT[wt],
          _vector("mean", mean, device, n, torch.float32), _vector("rstd", rstd, device, n, torch.float32), op, os_,
          dw.data_ptr() if want_dweight else None, db.data_ptr() if want_dbias else None, wp, wb, st)
    if want_dx and out is not None:
        _written(out)
    return dx, dw, db


RG_MAX_SIDE, RG_MAX_STEPS, RG_UPDATES_PER_LAUNCH = 16384, 32, 12


def _updates(grads, outs, weights=None, momenta=None, out_momenta=None):
    """The host array of rg_update over lists of matrices on one device, and their type."""
    assert len(grads) == len(outs) and all(x is None or len(x) == len(grads) for x in (weights, momenta, out_momenta)), "lists of one length are expected"
    u = (rg_update * max(len(grads), 1))()
    dt, device = (grads[0].dtype, grads[0].device) if grads else (torch.float32, None)
    for k, (e, g, o) in enumerate(zip(u, grads, outs)):
        e.rows, e.cols = g.shape
        e.grad, e.grad_stride = _rows("grad", g, device if k else None, None, dt)
        e.out, e.out_stride = _rows("out", o, device, g.shape, dt)
        if weights is not None:
            e.weight, e.weight_stride = _rows("weight", weights[k], device, g.shape, dt)
            e.momentum, e.momentum_stride = _rows("momentum", momenta[k], device, g.shape, torch.float32)
            e.momentum_out, e.momentum_out_stride = _rows("momentum", out_momenta[k], device, g.shape, torch.float32)
    return u, _ELEMENT[dt]


def _update_scratch(u, n, t, workspace, device, stream, *made):
    """(workspace address, its bytes, raw stream)."""
    mine = None
    if workspace is None:
        b = C.c_uint64()
        _call(device, lib().rg_update_workspace, u, n, t, C.byref(b))
        workspace = mine = torch.empty(max(b.value, 1), dtype=torch.uint8, device=device)
    p, size = _scratch(workspace, device)
    return p, size, _stream_and_use(device, stream, mine, *made), mine


def rg_update_workspace(matrices):
    """Bytes of scratch for an update of these matrices in one call."""
    if not matrices:
        return 0
    u, t = _updates(matrices, matrices)
    b = C.c_uint64()
    _call(matrices[0].device, lib().rg_update_workspace, u, len(matrices), t, C.byref(b))
    return b.value


def rg_orthogonalize(grads, steps=5, eps=1e-7, out=None, workspace=None, stream=None):
    """The orthogonalised form of every device matrix of the list.  out: a list of where they go (the matrices themselves: in place)."""
    if not grads:
        return [] if out is None else out
    made = out is None
    out = [torch.empty(g.shape, dtype=g.dtype, device=g.device) for g in grads] if made else out
    u, t = _updates(grads, out)
    device = grads[0].device
    p, b, st, _mine = _update_scratch(u, len(grads), t, workspace, device, stream, *(out if made else ()))
    _call(device, lib().rg_orthogonalize, u, len(grads), t, int(steps), eps, p, b, st)
    if not made:
        _written(*out)
    return out


def rg_muon_step(weights, grads, momenta, lr, weight_decay=0.0, momentum=0.95, nesterov=True, steps=5, eps=1e-7, out_weights=None, out_momenta=None,
                 workspace=None, stream=None):
    """One optimiser step on lists of device matrices; momenta are fp32.  In place, unless out_weights / out_momenta say where the new ones go."""
    out_weights = weights if out_weights is None else out_weights
    out_momenta = momenta if out_momenta is None else out_momenta
    u, t = _updates(grads, out_weights, weights, momenta, out_momenta)
    if not grads:
        return
    device = grads[0].device
    p, b, st, _mine = _update_scratch(u, len(grads), t, workspace, device, stream)
    _call(device, lib().rg_muon_step, u, len(grads), t, lr, weight_decay, momentum, 1 if nesterov else 0, int(steps), eps, p, b, st)
    _written(*out_weights, *out_momenta)


# ---------------------------------------------------------------- rows held in 8 bits, and the products on them
RG_MAX_HELD_COLS = 131072


def rg_rows8_bytes(cols):
    """Bytes of a held row of `cols` elements: its codes, zeros, its scale in the last four."""
    b = C.c_uint64()
    _check(lib().rg_rows8_bytes(int(cols), C.byref(b)))
    return b.value


def _held(name, t, device, cols):
    """(address, stride in bytes, rows) of held rows on `device` (any GPU, if None): a uint8 matrix of rg_rows8_bytes(cols) a row."""
    assert t.dim() == 2 and t.dtype == torch.uint8 and (t.is_cuda if device is None else t.device == device), f"{name}: expected a uint8 matrix on {device or 'the device'}"
    assert t.shape[1] == (cols + 19) // 16 * 16, f"{name}: rows of {t.shape[1]} bytes do not hold {cols} elements"
    along, across = t.stride()
    assert across == 1, f"{name}: the bytes of a row have to be contiguous"
    return t.data_ptr(), along, t.shape[0]


def _positions(rows, device):
    if rows is None:
        return None
    assert rows.device == device and rows.dtype == torch.int64 and rows.dim() == 1 and rows.is_contiguous(), f"rows: expected contiguous int64 positions on {device}"
    return rows.data_ptr()


def _made_scratch(device, entry, *args):
    """A workspace of the bytes that `entry` says, None where it says none."""
    b = C.c_uint64()
    _call(device, entry, *args, C.byref(b))
    return None if b.value == 0 else torch.empty(b.value, dtype=torch.uint8, device=device)


def _place(x, rows, out):
    """Where the result of rows that may lie in pinned host memory goes."""
    if x.is_cuda:
        return x.device
    assert x.is_pinned(), "expected device or pinned host memory"
    return out.device if out is not None else rows.device if rows is not None else torch.device("cuda", torch.cuda.current_device())


def rg_quantize_rows(x, rows=None, out=None, stream=None):
    """The rows of `x` (device or pinned matrix; rows may be padded), or those at the positions `rows` (int64; -1: a row of zeros), as
    held rows: a uint8 matrix of rg_rows8_bytes(x.shape[1]) a row.  out: where they go.  Pinned memory has to stay until the call's work on the device is done."""
    device = _place(x, rows, out)
    xp, xs = _rows("x", x, x.device if not x.is_cuda else None)
    n, d = x.shape
    n_out = n if rows is None else rows.shape[0]
    made = out is None
    if made:
        hs = (d + 19) // 16 * 16
        out = torch.empty((n_out, hs), dtype=torch.uint8, device=device)
        hp = out.data_ptr()
    else:
        hp, hs, got = _held("out", out, device, d)
        assert got == n_out, f"out: expected {n_out} rows, got {got}"
    st = _stream_and_use(device, stream, out if made else None)
    _call(device, lib().rg_quantize_rows, xp, xs, n, d, _ELEMENT[x.dtype], _positions(rows, device), n_out, hp, hs, st)
    if not made:
        _written(out)
    return out


def rg_dequantize_rows(held, cols, dtype=torch.float32, rows=None, out=None, stream=None):
    """What held rows of `cols` elements stand for, all of them or those at the positions `rows` (int64; -1: a row of zeros).  out: where it goes.  Pinned memory
    has to stay until the call's work on the device is done."""
    device = _place(held, rows, out)
    hp, hs, n = _held("held", held, held.device if not held.is_cuda else None, cols)
    n_out = n if rows is None else rows.shape[0]
    made = out is None
    if made:
        out = torch.empty((n_out, cols), dtype=dtype, device=device)
        op, os_ = out.data_ptr(), cols * dtype.itemsize
    else:
        dtype = out.dtype
        op, os_ = _rows("out", out, device, (n_out, cols))
    st = _stream_and_use(device, stream, out if made else None)
    _call(device, lib().rg_dequantize_rows, hp, hs, n, cols, _positions(rows, device), n_out, _ELEMENT[dtype], op, os_, st)
    if not made:
        _written(out)
    return out


def rg_rows8_product_workspace(n_rows, n_outs, cols, dtype=torch.float32):
    """Bytes of scratch that the product takes; dtype: of its result."""
    b = C.c_uint64()
    _check(lib().rg_rows8_product_workspace(int(n_rows), int(n_outs), int(cols), _ELEMENT[dtype], C.byref(b)))
    return b.value


def rg_rows8_product(x, w, cols, bias=None, dtype=torch.float32, out=None, workspace=None, stream=None):
    """x w^T + bias of held rows x and held weights w, both of `cols` elements a row; bias: fp32, or of the result's type.  out: where it
    goes; workspace: a device tensor of rg_rows8_product_workspace bytes, made here if None."""
    device = x.device
    xp, xs, n = _held("x", x, None, cols)
    wp, ws, m = _held("w", w, device, cols)
    made, mine = out is None, None
    if made:
        out = torch.empty((n, m), dtype=dtype, device=device)
        yp, ys = out.data_ptr(), m * out.element_size()
    else:
        yp, ys = _rows("out", out, device, (n, m))
        dtype = out.dtype
    bt = dtype if bias is None else bias.dtype
    bp = _vector("bias", bias, device, m, bt)
    if workspace is None:
        workspace = mine = _made_scratch(device, lib().rg_rows8_product_workspace, n, m, cols, _ELEMENT[dtype])
    sp, sb = (None, 0) if workspace is None else _scratch(workspace, device)
    st = _stream_and_use(device, stream, out if made else None, mine)
    _call(device, lib().rg_rows8_product, xp, xs, n, wp, ws, m, cols, bp, _ELEMENT[bt], yp, ys, _ELEMENT[dtype], sp, sb, st)
    if not made:
        _written(out)
    return out


def rg_rows8_product_backward_workspace(n_rows, n_outs, cols, dtype, want_dx=True, want_dweight=True, want_dbias=True):
    """Bytes of scratch that the backward pass takes."""
    b = C.c_uint64()
    _check(lib().rg_rows8_product_backward_workspace(int(n_rows), int(n_outs), int(cols), _ELEMENT[dtype], int(want_dx), int(want_dweight), int(want_dbias), C.byref(b)))
    return b.value


def rg_rows8_product_backward(dy, x, w, cols, want_dx=True, want_dweight=True, want_dbias=True, weight_dtype=None, out=None, workspace=None, stream=None):
    """(dx, dweight, dbias) of the product of held rows x and held weights w; None for what is not wanted.  x may be None where no dweight is, w where no dx
    is.  weight_dtype: of dweight and dbias, fp32 or dy's (the default).  out: where dx goes; workspace: a device tensor of rg_rows8_product_backward_workspace bytes, made here if None."""
    device, dt = dy.device, dy.dtype
    gp, gs = _rows("dy", dy, None)
    n, m = dy.shape
    wt = dt if weight_dtype is None else weight_dtype
    xp, xs, nx = (None, 0, n) if x is None else _held("x", x, device, cols)
    wp, ws, mw = (None, 0, m) if w is None else _held("w", w, device, cols)
    assert (nx, mw) == (n, m), f"dy of {n} x {m} does not belong to {nx} rows and {mw} weights"
    dx, op, os_, dw, db, mine = None, None, 0, None, None, None
    if want_dx:
        dx = torch.empty((n, cols), dtype=dt, device=device) if out is None else out
        op, os_ = _rows("out", dx, device, (n, cols), dt)
    if want_dweight:
        dw = torch.empty((m, cols), dtype=wt, device=device)
    if want_dbias:
        db = torch.empty(m, dtype=wt, device=device)
    if workspace is None:
        workspace = mine = _made_scratch(device, lib().rg_rows8_product_backward_workspace, n, m, cols, _ELEMENT[dt], int(want_dx), int(want_dweight), int(want_dbias))
    sp, sb = (None, 0) if workspace is None else _scratch(workspace, device)
    st = _stream_and_use(device, stream, dx if out is None else None, dw, db, mine)
    _call(device, lib().rg_rows8_product_backward, gp, gs, xp, xs, wp, ws, n, m, cols, _ELEMENT[dt], op, os_, dw.data_ptr() if want_dweight else None,
          cols * wt.itemsize, db.data_ptr() if want_dbias else None, _ELEMENT[wt], sp, sb, st)
    if want_dx and out is not None:
        _written(dx)
    return dx, dw, db


def rg_trim_memory():
    """Return the library's cached device blocks to the driver."""
    lib().rg_trim_memory()


def rg_profile_enable(on=True):
    lib().rg_profile_enable(1 if on else 0)


def rg_profile_reset():
    lib().rg_profile_reset()


def rg_profile_read():
    ms = (C.c_double * len(KERNEL_GROUPS))()
    n = (C.c_uint64 * len(KERNEL_GROUPS))()
    _check(lib().rg_profile_read(ms, n))
    return {g: dict(ms=ms[i], launches=int(n[i])) for i, g in enumerate(KERNEL_GROUPS)}


class TorchAllocator:
    """rg_allocator backed by torch: device buffers from the caching allocator, pinned buffers from pinned tensors.
    limit_bytes: requests above it are refused (NULL to the library), as an allocator that has run out would."""

    def __init__(self, limit_bytes=None):
        self.live = {}
        self.n_alloc = 0
        self.n_refused = 0

        def _alloc(nbytes, kind, _ctx):
            if limit_bytes is not None and int(nbytes) > limit_bytes:
                self.n_refused += 1
                return None
            try:
                if kind == 1:
                    t = torch.empty(int(nbytes), dtype=torch.uint8, device="cuda")
                else:
                    t = torch.empty(int(nbytes), dtype=torch.uint8, pin_memory=True)
            except Exception:       # noqa: BLE001 -- report failure to the library as NULL
                return None
            self.live[t.data_ptr()] = t
            self.n_alloc += 1
            return t.data_ptr()

        def _free(p, _kind, _ctx):
            self.live.pop(p, None)

        self._a, self._f = ALLOC_FN(_alloc), FREE_FN(_free)
        self.struct = rg_allocator(self._a, self._f, None)
