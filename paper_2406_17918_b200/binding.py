"""ctypes binding of ``libgs.so``: argument marshalling only.

Functions keep the names and argument order of ``include/gs.h``.  Device buffers are torch CUDA
tensors (torch is used for device memory and streams only); the binding passes their
``data_ptr()`` and keeps them alive on the small Python handle objects.
"""
from __future__ import annotations

import ctypes
import math
import os
import re
from array import array

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libgs.so")
_HEADER = os.path.join(os.path.dirname(_HERE), "include", "gs.h")

GS_MODE_FCR, GS_MODE_OTF, GS_MODE_FBL, GS_MODE_OTF_FETCH = 0, 1, 2, 3
GS_F32, GS_BF16 = 0, 1
GS_DEDUP_DIRECT, GS_DEDUP_HASH, GS_DEDUP_SORT, GS_DEDUP_AUTO = 0, 1, 2, 3
GS_MAX_HOPS = 8
COUNTS_READBACK_BYTES = 4 * (1 + (GS_MAX_HOPS + 1) + GS_MAX_HOPS)  # status + n_k + m_k, what gs_batch_counts copies

_STATUS_NAMES = {0: "GS_OK", 1: "GS_ERR_ARG", 2: "GS_ERR_ALIGN", 3: "GS_ERR_RANGE", 4: "GS_ERR_WORKSPACE",
                 5: "GS_ERR_DUP_SEED", 6: "GS_ERR_CUDA"}


class GsError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("%s: %s" % (_STATUS_NAMES.get(status, status), message))
        self.status = status


class _CBlock(ctypes.Structure):
    _fields_ = [("max_dst", ctypes.c_int32), ("max_src", ctypes.c_int32), ("max_edges", ctypes.c_int32),
                ("d_num_dst", ctypes.c_void_p), ("d_num_src", ctypes.c_void_p), ("d_num_edges", ctypes.c_void_p),
                ("d_indptr", ctypes.c_void_p), ("d_indices", ctypes.c_void_p)]


class _CBlockBuffers(ctypes.Structure):
    _fields_ = [("d_indptr", ctypes.c_void_p), ("indptr_capacity", ctypes.c_int64),
                ("d_indices", ctypes.c_void_p), ("indices_capacity", ctypes.c_int64)]


NOALLOC_SCRATCH_BYTES = 64 << 20


def library_path() -> str:
    return _LIB_PATH


def exported_symbols():
    """Names of the functions ``include/gs.h`` declares."""
    text = open(_HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(gs_[a-z_]+)\s*\(", text)))


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError("%s is missing: run `python -m paper_2406_17918_b200.build` "
                          "(there is no CPU fallback)" % _LIB_PATH)
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, u32, u64, dbl, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                                       ctypes.c_uint64, ctypes.c_double, ctypes.c_size_t)
    pvp = ctypes.POINTER(vp)
    psz = ctypes.POINTER(sz)
    sig = {
        "gs_graph_create": [i64, i64, vp, vp, vp, ctypes.c_int, i32, i64, pvp],
        "gs_graph_validate": [vp, vp, ctypes.POINTER(i64)],
        "gs_graph_set_gather_grid": [vp, i32],
        "gs_gather_status": [vp],
        "gs_cache_bytes": [vp, i32, i32, i32, psz],
        "gs_workspace_bytes": [vp, i32, vp, i32, psz],
        "gs_cache_init": [vp, i32, vp, i32, u64, i32, vp, sz, vp, pvp],
        "gs_cache_refresh_all": [vp, ctypes.c_int, ctypes.c_double, ctypes.c_uint32, vp],
        "gs_cache_bytes_split": [vp, i32, i32, i32, i64, psz],
        "gs_cache_init_split": [vp, i32, vp, i32, u64, i32, i32, i64, vp, sz, vp, pvp],
        "gs_sample_batch": [vp, vp, i32, ctypes.c_int, dbl, u32, vp, sz, vp, vp, pvp, pvp],
        "gs_sample_batch_host": [vp, vp, i32, ctypes.c_int, dbl, u32, vp, sz, vp, vp, pvp, vp, vp],
        "gs_sample_batch_noalloc": [vp, vp, i32, ctypes.c_int, dbl, u32, vp, i64, vp, vp, vp, pvp],
        "gs_batch_counts": [vp, vp, vp, vp],
        "gs_gather_features": [vp, vp, vp, i32, vp, i64, vp],
        "gs_cache_read_rows": [vp, i32, vp, i32, vp, vp],
        "gs_cache_export_bytes": [vp, psz],
        "gs_cache_export": [vp, vp, sz, vp],
        "gs_cache_import": [vp, vp, sz, vp],
        "gs_sync_status": [vp, vp],
        "gs_gather_rows": [vp, ctypes.c_int, i32, i64, i64, i64, vp, vp, i32, vp, i64, vp],
        "gs_gather_rows_peer": [vp, i32, i64, ctypes.c_int, i32, i64, vp, vp, i32, vp, i64, vp],
        "gs_shard_bucket": [vp, i32, i64, i32, vp, vp, vp, vp],
        "gs_shard_bucket_counted": [vp, vp, i32, i64, i32, vp, vp, vp, vp],
        "gs_shard_workspace_bytes": [vp, i32, i32, psz],
        "gs_shard_bucket_fixed": [vp, vp, i32, i64, i32, i32, vp, vp, vp, vp],
        "gs_shard_sample_rows": [vp, vp, i32, i32, ctypes.c_int, dbl, u32, vp, sz, vp, vp],
        "gs_shard_sample_rows_counted": [vp, vp, vp, i32, i32, ctypes.c_int, dbl, u32, vp, sz, vp, vp],
        "gs_shard_status": [vp, vp],
        "gs_shard_merge": [vp, vp, i32, i32, i64, i64, vp, vp, vp, vp],
        "gs_shard_fan_out": [vp, vp, i32, i32, i64, i64, vp, vp, vp, vp, i32, vp, vp],
        "gs_shard_extend": [vp, i32, vp, i32, vp, vp, vp, sz, vp, vp, pvp],
        "gs_shard_extend_fixed": [vp, i32, vp, i32, vp, i32, vp, vp, sz, vp, vp, pvp],
        "gs_batch_stats": [vp, vp, vp],
        "gs_cache_profile_begin": [vp, i32],
        "gs_cache_profile_end": [vp, vp, vp, vp],
        "gs_cache_set_tuning": [vp, dbl, dbl, i32],
        "gs_debug_set_grid_cap": [i32],
        "gs_alu_ceiling": [i32, i32, vp, ctypes.POINTER(dbl)],
        "gs_cache_set_dedup": [vp, i32],
        "gs_graph_count_dense": [vp, i32, vp, ctypes.POINTER(i64)],
        "gs_embedding_lookup": [vp, ctypes.c_int, i64, i32, i64, vp, vp, i32, ctypes.c_float, vp, ctypes.c_int, i64, vp],
        "gs_embedding_workspace_bytes": [i32, i64, i32, psz],
        "gs_embedding_backward": [vp, ctypes.c_int, i64, vp, vp, i32, i64, i32, ctypes.c_float, vp, ctypes.c_int, i64, vp, sz, vp],
        "gs_embedding_backward_sparse": [vp, ctypes.c_int, i64, vp, vp, i32, i64, i32, ctypes.c_float, vp, vp, vp, ctypes.c_int, i64,
                                         vp, sz, vp],
        "gs_train_status": [vp],
        "gs_xent_workspace_bytes": [i32, i64, i32, ctypes.c_int, psz],
        "gs_xent_forward": [vp, i64, vp, i64, ctypes.c_int, i32, i64, i32, ctypes.c_float, vp, vp, vp, vp, sz, vp],
        "gs_xent_backward": [vp, i64, vp, i64, ctypes.c_int, i32, i64, i32, ctypes.c_float, vp, vp, vp, vp, i64, vp, i64, ctypes.c_int, vp, sz, vp],
        "gs_block_attention_workspace_bytes": [i32, i32, i32, i32, psz],
        "gs_block_attention_forward": [vp, i32, ctypes.c_int, i32, i32, i32, ctypes.c_float, vp, vp, vp, vp, vp, vp, sz, vp],
        "gs_block_reverse": [vp, vp, vp, vp, vp, sz, vp],
        "gs_block_attention_backward": [vp, i32, vp, vp, vp, ctypes.c_int, i32, i32, i32, ctypes.c_float, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                        vp, sz, vp],
        "gs_rms_norm_workspace_bytes": [i32, i32, psz],
        "gs_rms_norm_forward": [vp, i64, vp, i64, ctypes.c_int, vp, ctypes.c_int, vp, i32, i32, ctypes.c_float, vp, i64, vp, i64, vp],
        "gs_rms_norm_coded": [vp, i64, vp, i64, ctypes.c_int, vp, ctypes.c_int, vp, i32, i32, ctypes.c_float, vp, i64, vp, vp],
        "gs_rms_norm_backward": [vp, i64, vp, i64, vp, i64, ctypes.c_int, vp, ctypes.c_int, vp, i32, i32, ctypes.c_float, vp, i64, vp, vp, sz, vp],
        "gs_coded_write": [vp, ctypes.c_int, vp, vp, i64, vp, i32, vp, vp],
        "gs_coded_read": [vp, vp, i64, vp, i32, ctypes.c_int, vp, vp],
        "gs_coded_attention_workspace_bytes": [i32, i32, i32, psz],
        "gs_coded_attention_forward": [vp, vp, i32, ctypes.c_int, i32, i32, ctypes.c_float, vp, vp, vp, vp, vp, vp, sz, vp],
        "gs_grad_workspace_bytes": [i32, psz],
        "gs_grad_norm": [vp, i32, vp, vp, sz, vp],
        "gs_grad_clip": [vp, i32, ctypes.c_float, vp, vp, sz, vp],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    L.gs_graph_destroy.argtypes = [vp]
    L.gs_graph_destroy.restype = None
    L.gs_cache_destroy.argtypes = [vp]
    L.gs_cache_destroy.restype = None
    L.gs_last_error.argtypes = []
    L.gs_last_error.restype = ctypes.c_char_p
    L.gs_stats_word_offset.argtypes = []
    L.gs_stats_word_offset.restype = ctypes.c_int32
    L.gs_kernel_launches.argtypes = []
    L.gs_kernel_launches.restype = ctypes.c_int64
    return L


_L = _load()


def gs_stats_word_offset() -> int:
    return int(_L.gs_stats_word_offset())


def gs_last_error() -> str:
    return _L.gs_last_error().decode()


def gs_kernel_launches() -> int:
    return int(_L.gs_kernel_launches())


def _check(status):
    if status != 0:
        raise GsError(status, gs_last_error())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _i32_array(values):
    return (ctypes.c_int32 * len(values))(*[int(v) for v in values])


class Graph:
    """Handle of gs_graph plus references that keep the borrowed tensors alive."""

    def __init__(self, handle, indptr, indices, features, dtype, feat_dim):
        self.handle, self.indptr, self.indices, self.features = handle, indptr, indices, features
        self.dtype, self.feat_dim = dtype, feat_dim
        self.num_nodes = indptr.numel() - 1

    def close(self):
        if self.handle:
            _L.gs_graph_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Cache:
    def __init__(self, handle, graph, storage, fanouts, cache_width, shared):
        self.handle, self.graph, self.storage = handle, graph, storage
        self.fanouts, self.cache_width, self.shared = list(fanouts), cache_width, bool(shared)
        self.num_hops = len(self.fanouts)

    def close(self):
        if self.handle:
            _L.gs_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Block:
    """Device view of one hop's block; tensors alias the workspace (no copies)."""

    def __init__(self, cb: _CBlock, workspace: torch.Tensor, header: torch.Tensor):
        self.max_dst, self.max_src, self.max_edges = cb.max_dst, cb.max_src, cb.max_edges
        self._ws, self._hdr = workspace, header
        self._indptr_off = cb.d_indptr - workspace.data_ptr()
        self._indices_off = cb.d_indices - workspace.data_ptr()
        hp = header.data_ptr()
        self._cnt = ((cb.d_num_dst - hp) // 4, (cb.d_num_src - hp) // 4, (cb.d_num_edges - hp) // 4)

    def count_words(self):
        """int32 word positions of (num_dst, num_src, num_edges) inside the cache storage."""
        return self._cnt

    def counts_device(self):
        """(num_dst, num_src, num_edges) as 0-d device tensors aliasing the cache's state header."""
        h = self._hdr.view(torch.int32)
        return tuple(h[i] for i in self._cnt)

    def indptr(self, num_dst: int) -> torch.Tensor:
        return self._ws[self._indptr_off:self._indptr_off + 4 * (num_dst + 1)].view(torch.int32)

    def indices(self, num_edges: int) -> torch.Tensor:
        return self._ws[self._indices_off:self._indices_off + 4 * num_edges].view(torch.int32)


def gs_graph_create(indptr: torch.Tensor, indices: torch.Tensor, features, dtype=None) -> Graph:
    if indptr.dtype != torch.int64 or indices.dtype != torch.int32:
        raise TypeError("indptr must be int64 and indices int32")
    if not (indptr.is_cuda and indices.is_cuda and indptr.is_contiguous() and indices.is_contiguous()):
        raise ValueError("indptr/indices must be contiguous CUDA tensors")
    feat_dim, feat_ld = 0, 0
    if features is not None:
        if not features.is_cuda or features.dim() != 2 or features.stride(1) != 1:
            raise ValueError("features must be a row-major 2-D CUDA tensor")
        dtype = {torch.float32: GS_F32, torch.bfloat16: GS_BF16}[features.dtype]
        feat_dim, feat_ld = features.shape[1], features.stride(0)
    elif dtype is None:
        dtype = GS_F32
    h = ctypes.c_void_p()
    _check(_L.gs_graph_create(indptr.numel() - 1, indices.numel(), _ptr(indptr), _ptr(indices), _ptr(features),
                              dtype, feat_dim, feat_ld, ctypes.byref(h)))
    return Graph(h, indptr, indices, features, dtype, feat_dim)


def gs_graph_set_gather_grid(graph: Graph, blocks_per_sm: int):
    _check(_L.gs_graph_set_gather_grid(graph.handle, int(blocks_per_sm)))


def gs_gather_status(stream=None):
    """Synchronises; raises if a bulk-copy gather ever gave up waiting."""
    _check(_L.gs_gather_status(_stream(stream)))


def gs_graph_validate(graph: Graph, stream=None) -> int:
    """Checks the CSR contract on the device; returns -1, or raises GsError naming the first bad row."""
    bad = ctypes.c_int64(-1)
    _check(_L.gs_graph_validate(graph.handle, _stream(stream), ctypes.byref(bad)))
    return int(bad.value)


def gs_cache_bytes(graph: Graph, num_hops: int, cache_width: int, shared: bool) -> int:
    out = ctypes.c_size_t()
    _check(_L.gs_cache_bytes(graph.handle, num_hops, cache_width, int(shared), ctypes.byref(out)))
    return out.value


def gs_workspace_bytes(graph: Graph, fanouts, max_seeds: int) -> int:
    out = ctypes.c_size_t()
    _check(_L.gs_workspace_bytes(graph.handle, len(fanouts), _i32_array(fanouts), max_seeds, ctypes.byref(out)))
    return out.value


def gs_cache_init(graph: Graph, fanouts, cache_width: int, seed: int, shared: bool, storage: torch.Tensor = None,
                  stream=None) -> Cache:
    if storage is None:
        storage = torch.empty(gs_cache_bytes(graph, len(fanouts), cache_width, shared), dtype=torch.uint8,
                              device=graph.indptr.device)
    h = ctypes.c_void_p()
    _check(_L.gs_cache_init(graph.handle, len(fanouts), _i32_array(fanouts), cache_width, ctypes.c_uint64(seed),
                            int(shared), _ptr(storage), storage.numel(), _stream(stream), ctypes.byref(h)))
    return Cache(h, graph, storage, fanouts, cache_width, shared)


def gs_cache_bytes_split(graph: Graph, num_hops: int, cache_width: int, shared: bool, dense_rows: int) -> int:
    out = ctypes.c_size_t()
    _check(_L.gs_cache_bytes_split(graph.handle, num_hops, cache_width, int(shared), dense_rows, ctypes.byref(out)))
    return out.value


def gs_graph_count_dense(graph: Graph, theta: int, stream=None) -> int:
    """Nodes with degree > theta, counted by the library (synchronises)."""
    out = ctypes.c_int64()
    _check(_L.gs_graph_count_dense(graph.handle, int(theta), _stream(stream), ctypes.byref(out)))
    return int(out.value)


def gs_cache_init_split(graph: Graph, fanouts, cache_width: int, seed: int, shared: bool, theta: int,
                        dense_rows: int = None, storage: torch.Tensor = None, stream=None) -> Cache:
    """Cache rows only for nodes with degree > theta; the others are sampled from the graph."""
    if dense_rows is None:
        dense_rows = gs_graph_count_dense(graph, theta, stream)
    if storage is None:
        storage = torch.empty(gs_cache_bytes_split(graph, len(fanouts), cache_width, shared, dense_rows),
                              dtype=torch.uint8, device=graph.indptr.device)
    h = ctypes.c_void_p()
    _check(_L.gs_cache_init_split(graph.handle, len(fanouts), _i32_array(fanouts), cache_width, ctypes.c_uint64(seed),
                                  int(shared), int(theta), int(dense_rows), _ptr(storage), storage.numel(),
                                  _stream(stream), ctypes.byref(h)))
    return Cache(h, graph, storage, fanouts, cache_width, shared)


def gs_cache_refresh_all(cache: Cache, mode: int, gamma: float, step: int, stream=None) -> None:
    """Refresh every cached row of every layer (the periodic-refresh branch of Algorithms 2 and 3)."""
    _check(_L.gs_cache_refresh_all(cache.handle, mode, float(gamma), step, _stream(stream)))


def _blocks_out(cache: Cache, cblocks, workspace):
    return [Block(cblocks[l], workspace, cache.storage) for l in range(cache.num_hops)]


def gs_sample_batch(cache: Cache, seeds: torch.Tensor, mode: int, gamma: float, step: int, workspace: torch.Tensor,
                    stream=None):
    """Returns (blocks by layer, input_nodes tensor of capacity max_src, device count tensor)."""
    if seeds.dtype != torch.int32 or not seeds.is_cuda or not seeds.is_contiguous():
        raise TypeError("seeds must be a contiguous int32 CUDA tensor")
    cblocks = (_CBlock * cache.num_hops)()
    d_in, d_cnt = ctypes.c_void_p(), ctypes.c_void_p()
    _check(_L.gs_sample_batch(cache.handle, _ptr(seeds), seeds.numel(), mode, float(gamma), step, _ptr(workspace),
                              workspace.numel(), _stream(stream), cblocks, ctypes.byref(d_in), ctypes.byref(d_cnt)))
    blocks = _blocks_out(cache, cblocks, workspace)
    off = d_in.value - workspace.data_ptr()
    input_nodes = workspace[off:off + 4 * blocks[0].max_src].view(torch.int32)
    cnt_index = (d_cnt.value - cache.storage.data_ptr()) // 4
    return blocks, input_nodes, cache.storage.view(torch.int32)[cnt_index]


def gs_sample_batch_host(cache: Cache, seeds_host: torch.Tensor, mode: int, gamma: float, step: int,
                         workspace: torch.Tensor, stream=None):
    """Seeds in (pinned) host memory; synchronises.  Returns (blocks, input_nodes, n list, m list)."""
    if seeds_host.dtype != torch.int32 or seeds_host.is_cuda or not seeds_host.is_contiguous():
        raise TypeError("seeds_host must be a contiguous int32 CPU tensor")
    cblocks = (_CBlock * cache.num_hops)()
    d_in = ctypes.c_void_p()
    n = (ctypes.c_int32 * (cache.num_hops + 1))()
    m = (ctypes.c_int32 * cache.num_hops)()
    _check(_L.gs_sample_batch_host(cache.handle, _ptr(seeds_host), seeds_host.numel(), mode, float(gamma), step,
                                   _ptr(workspace), workspace.numel(), _stream(stream), cblocks, ctypes.byref(d_in),
                                   n, m))
    blocks = _blocks_out(cache, cblocks, workspace)
    off = d_in.value - workspace.data_ptr()
    input_nodes = workspace[off:off + 4 * blocks[0].max_src].view(torch.int32)
    return blocks, input_nodes, list(n), list(m)


class OutBlock:
    """One hop's block as written by gs_sample_batch_noalloc into the caller's tensors."""

    def __init__(self, cb, indptr, indices):
        self.max_dst, self.max_src, self.max_edges = cb.max_dst, cb.max_src, cb.max_edges
        self._indptr, self._indices = indptr, indices

    def indptr(self, num_dst: int) -> torch.Tensor:
        return self._indptr[: num_dst + 1]

    def indices(self, num_edges: int) -> torch.Tensor:
        return self._indices[:num_edges]


def gs_sample_batch_noalloc(cache: Cache, seeds: torch.Tensor, mode: int, gamma: float, step: int,
                            input_nodes: torch.Tensor, indptr_bufs, indices_bufs, stream=None):
    """The batch call for callers that may not allocate device memory: scratch is the library's
    built-in array, results land in the int32 CUDA tensors passed here (`indptr_bufs[l]`,
    `indices_bufs[l]` by layer, and `input_nodes`).  Nothing is allocated by this function either.
    Returns the blocks (views of the caller's tensors), by layer."""
    if seeds.dtype != torch.int32 or not seeds.is_cuda or not seeds.is_contiguous():
        raise TypeError("seeds must be a contiguous int32 CUDA tensor")
    bufs = (_CBlockBuffers * cache.num_hops)()
    for l in range(cache.num_hops):
        for t in (indptr_bufs[l], indices_bufs[l]):
            if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
                raise TypeError("block buffers must be contiguous int32 CUDA tensors")
        bufs[l].d_indptr, bufs[l].indptr_capacity = indptr_bufs[l].data_ptr(), indptr_bufs[l].numel()
        bufs[l].d_indices, bufs[l].indices_capacity = indices_bufs[l].data_ptr(), indices_bufs[l].numel()
    cblocks = (_CBlock * cache.num_hops)()
    d_cnt = ctypes.c_void_p()
    _check(_L.gs_sample_batch_noalloc(cache.handle, _ptr(seeds), seeds.numel(), mode, float(gamma), step,
                                      _ptr(input_nodes), input_nodes.numel(), bufs, _stream(stream), cblocks,
                                      ctypes.byref(d_cnt)))
    return [OutBlock(cblocks[l], indptr_bufs[l], indices_bufs[l]) for l in range(cache.num_hops)]


def gs_batch_counts(cache: Cache, stream=None):
    """Synchronises; returns ([n_0..n_L] by sampling step, [edges per block] by layer)."""
    n = (ctypes.c_int32 * (cache.num_hops + 1))()
    m = (ctypes.c_int32 * cache.num_hops)()
    _check(_L.gs_batch_counts(cache.handle, _stream(stream), n, m))
    return list(n), list(m)


def gs_gather_features(graph: Graph, ids: torch.Tensor, count, out: torch.Tensor, stream=None):
    """count: a 0-d int32 CUDA tensor (device scalar) or None to gather out.shape[0] rows."""
    if ids.dtype != torch.int32 or not ids.is_cuda:
        raise TypeError("ids must be an int32 CUDA tensor")
    if out.dim() != 2 or out.stride(1) != 1 or out.dtype != graph.features.dtype:
        raise TypeError("out must be a row-major 2-D tensor of the feature dtype")
    bound = min(out.shape[0], ids.numel())
    _check(_L.gs_gather_features(graph.handle, _ptr(ids), _ptr(count), bound, _ptr(out), out.stride(0),
                                 _stream(stream)))
    return out


def gs_gather_rows(src: torch.Tensor, ids: torch.Tensor, out: torch.Tensor, first_row: int = 0, count=None, stream=None):
    """out[i] = src[ids[i] - first_row] for a row-major 2-D f32 / bf16 CUDA tensor."""
    if src.dim() != 2 or src.stride(1) != 1 or out.dim() != 2 or out.stride(1) != 1 or out.dtype != src.dtype:
        raise TypeError("src and out must be row-major 2-D tensors of one dtype")
    if ids.dtype != torch.int32 or not ids.is_cuda:
        raise TypeError("ids must be an int32 CUDA tensor")
    dtype = {torch.float32: GS_F32, torch.bfloat16: GS_BF16}[src.dtype]
    bound = min(out.shape[0], ids.numel())
    _check(_L.gs_gather_rows(_ptr(src), dtype, src.shape[1], src.stride(0), int(first_row), src.shape[0], _ptr(ids), _ptr(count), bound,
                             _ptr(out), out.stride(0), _stream(stream)))
    return out


def gs_gather_rows_peer(shard_bases, num_rows: int, dtype: torch.dtype, row_elems: int, src_ld: int, ids: torch.Tensor,
                        out: torch.Tensor, count=None, stream=None):
    """out[i] = row ids[i] of a matrix split over len(shard_bases) row shards; `shard_bases` are device
    addresses (ints), local or peer-mapped.  One kernel: the rows are pulled straight from their owners."""
    if ids.dtype != torch.int32 or not ids.is_cuda:
        raise TypeError("ids must be an int32 CUDA tensor")
    if out.dim() != 2 or out.stride(1) != 1 or out.dtype != dtype:
        raise TypeError("out must be a row-major 2-D tensor of the given dtype")
    world = len(shard_bases)
    arr = (ctypes.c_void_p * world)(*[ctypes.c_void_p(int(b)) for b in shard_bases])
    bound = min(out.shape[0], ids.numel())
    _check(_L.gs_gather_rows_peer(arr, world, int(num_rows), {torch.float32: GS_F32, torch.bfloat16: GS_BF16}[dtype],
                                  int(row_elems), int(src_ld), _ptr(ids), _ptr(count), bound, _ptr(out), out.stride(0),
                                  _stream(stream)))
    return out


def gs_shard_bucket(nodes: torch.Tensor, num_nodes: int, world: int, stream=None, count=None, capacity=None, out=None):
    """Group node ids by owner.  Returns (sorted ids, slot of every input id, int32[2*world+1] device counts).
    `count`: a 0-d int32 CUDA tensor with the list's length when only the device knows it (`nodes` is then the bound).
    `capacity`: every owner's group gets a segment of that many ids (sorted ids: world*capacity entries) instead of
    the groups being packed.  `out`: (sorted, slot, counts) tensors to write into instead of new ones."""
    if nodes.dtype != torch.int32 or not nodes.is_cuda or not nodes.is_contiguous():
        raise TypeError("nodes must be a contiguous int32 CUDA tensor")
    if out is not None:
        sorted_ids, slot, counts = out
        need = nodes.numel() if capacity is None else world * int(capacity)
        if sorted_ids.numel() < need or slot.numel() < nodes.numel() or counts.numel() < 2 * world + 1:
            raise ValueError("an output tensor is too small")
        for t in out:
            if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
                raise TypeError("outputs must be contiguous int32 CUDA tensors")
    else:
        sorted_ids = torch.empty_like(nodes) if capacity is None else torch.empty(world * int(capacity), dtype=torch.int32, device=nodes.device)
        slot = torch.empty_like(nodes)
        counts = torch.empty(2 * world + 1, dtype=torch.int32, device=nodes.device)
    if capacity is not None:
        _check(_L.gs_shard_bucket_fixed(_ptr(nodes), _ptr(count), nodes.numel(), int(num_nodes), int(world), int(capacity),
                                        _ptr(sorted_ids), _ptr(slot), _ptr(counts), _stream(stream)))
    elif count is None:
        _check(_L.gs_shard_bucket(_ptr(nodes), nodes.numel(), int(num_nodes), int(world), _ptr(sorted_ids), _ptr(slot),
                                  _ptr(counts), _stream(stream)))
    else:
        _check(_L.gs_shard_bucket_counted(_ptr(nodes), _ptr(count), nodes.numel(), int(num_nodes), int(world),
                                          _ptr(sorted_ids), _ptr(slot), _ptr(counts), _stream(stream)))
    return sorted_ids, slot, counts


def gs_shard_workspace_bytes(graph: Graph, fanout: int, max_nodes: int) -> int:
    out = ctypes.c_size_t()
    _check(_L.gs_shard_workspace_bytes(graph.handle, int(fanout), int(max_nodes), ctypes.byref(out)))
    return out.value


def gs_shard_sample_rows(cache: Cache, nodes: torch.Tensor, layer: int, mode: int, rate: float, step: int,
                         workspace: torch.Tensor, picks: torch.Tensor = None, stream=None, count=None) -> torch.Tensor:
    """Owner side of one hop: picks[n, fanout(layer)] (-1 padded) for n distinct nodes of this shard.
    `count`: a 0-d / 1-element int32 CUDA tensor with the list's length (`nodes` is then the bound; only that
    many rows of `picks` are written)."""
    if nodes.dtype != torch.int32 or not nodes.is_cuda or not nodes.is_contiguous():
        raise TypeError("nodes must be a contiguous int32 CUDA tensor")
    f = cache.fanouts[layer] if 0 <= layer < cache.num_hops else 1     # a bad layer is reported by the library
    if picks is None:
        picks = torch.empty((nodes.numel(), f), dtype=torch.int32, device=nodes.device)
    elif picks.dtype != torch.int32 or not picks.is_contiguous() or picks.numel() < nodes.numel() * f:
        raise TypeError("picks must be a contiguous int32 tensor of at least [len(nodes), fanout]")
    if count is None:
        _check(_L.gs_shard_sample_rows(cache.handle, _ptr(nodes), nodes.numel(), int(layer), mode, float(rate), step,
                                       _ptr(workspace), workspace.numel(), _stream(stream), _ptr(picks)))
    else:
        _check(_L.gs_shard_sample_rows_counted(cache.handle, _ptr(nodes), _ptr(count), nodes.numel(), int(layer), mode,
                                               float(rate), step, _ptr(workspace), workspace.numel(), _stream(stream),
                                               _ptr(picks)))
    return picks


def _i32_cuda(*tensors):
    for t in tensors:
        if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
            raise TypeError("contiguous int32 CUDA tensors expected")


def gs_shard_merge(lists: torch.Tensor, counts: torch.Tensor, world: int, first_row: int, index: torch.Tensor,
                   distinct: torch.Tensor, num_distinct: torch.Tensor, stream=None):
    """Owner side: one place in `distinct` for every node any of the `world` fixed-pitch lists asks for.
    index: int32[rows owned], all -1 between batches; num_distinct: int32[2] (count, status word)."""
    _i32_cuda(lists, counts, index, distinct, num_distinct)
    capacity = lists.numel() // int(world)
    if lists.numel() != capacity * world or counts.numel() < world or num_distinct.numel() < 2 or \
            distinct.numel() < min(lists.numel(), index.numel()):
        raise ValueError("bad tensor sizes")
    _check(_L.gs_shard_merge(_ptr(lists), _ptr(counts), int(world), capacity, int(first_row), index.numel(), _ptr(index),
                             _ptr(distinct), _ptr(num_distinct), _stream(stream)))
    return distinct, num_distinct


def gs_shard_fan_out(lists: torch.Tensor, counts: torch.Tensor, world: int, first_row: int, index: torch.Tensor,
                     distinct: torch.Tensor, num_distinct: torch.Tensor, rows: torch.Tensor, out: torch.Tensor, stream=None):
    """out[e] = rows[place of lists[e]] for every entry of every list; puts `index` back to all -1."""
    _i32_cuda(lists, counts, index, distinct, num_distinct, rows, out)
    capacity = lists.numel() // int(world)
    f = rows.shape[1]
    if out.numel() < lists.numel() * f or rows.shape[0] < min(lists.numel(), index.numel()) or distinct.numel() < min(lists.numel(), index.numel()):
        raise ValueError("bad tensor sizes")
    _check(_L.gs_shard_fan_out(_ptr(lists), _ptr(counts), int(world), capacity, int(first_row), index.numel(), _ptr(index),
                               _ptr(distinct), _ptr(num_distinct), _ptr(rows), int(f), _ptr(out), _stream(stream)))
    return out


def gs_shard_status(cache: Cache, stream=None):
    _check(_L.gs_shard_status(cache.handle, _stream(stream)))


def gs_shard_extend(cache: Cache, k: int, seeds, reply: torch.Tensor, slot: torch.Tensor, workspace: torch.Tensor,
                    stream=None, reply_rows=None):
    """Requester side of hop k.  Returns (block of layer L-1-k, frontier array aliasing the workspace).
    `reply_rows`: rows of a fixed-pitch reply (world * capacity, see gs_shard_bucket)."""
    cb = _CBlock()
    d_fr = ctypes.c_void_p()
    if reply_rows is None:
        _check(_L.gs_shard_extend(cache.handle, int(k), _ptr(seeds), 0 if seeds is None else seeds.numel(), _ptr(reply),
                                  _ptr(slot), _ptr(workspace), workspace.numel(), _stream(stream), ctypes.byref(cb),
                                  ctypes.byref(d_fr)))
    else:
        if 0 <= k < cache.num_hops and reply.numel() < int(reply_rows) * cache.fanouts[cache.num_hops - 1 - k]:
            raise ValueError("reply holds fewer than reply_rows rows")
        _check(_L.gs_shard_extend_fixed(cache.handle, int(k), _ptr(seeds), 0 if seeds is None else seeds.numel(), _ptr(reply),
                                        int(reply_rows), _ptr(slot), _ptr(workspace), workspace.numel(), _stream(stream),
                                        ctypes.byref(cb), ctypes.byref(d_fr)))
    block = Block(cb, workspace, cache.storage)
    off = d_fr.value - workspace.data_ptr()
    return block, workspace[off:off + 4 * block.max_src].view(torch.int32)


def gs_cache_read_rows(cache: Cache, layer: int, nodes: torch.Tensor, stream=None) -> torch.Tensor:
    out = torch.empty((nodes.numel(), cache.cache_width), dtype=torch.int32, device=nodes.device)
    _check(_L.gs_cache_read_rows(cache.handle, layer, _ptr(nodes), nodes.numel(), _ptr(out), _stream(stream)))
    return out


def gs_cache_export(cache: Cache, stream=None) -> torch.Tensor:
    nbytes = ctypes.c_size_t()
    _check(_L.gs_cache_export_bytes(cache.handle, ctypes.byref(nbytes)))
    blob = torch.empty(nbytes.value, dtype=torch.uint8, device=cache.storage.device)
    _check(_L.gs_cache_export(cache.handle, _ptr(blob), blob.numel(), _stream(stream)))
    return blob


def gs_cache_import(cache: Cache, blob: torch.Tensor, stream=None):
    _check(_L.gs_cache_import(cache.handle, _ptr(blob), blob.numel(), _stream(stream)))


def gs_batch_stats(cache: Cache, stream=None):
    """Synchronises; {'slow_refills': ..., 'queued_rescans': ...} of the last batch."""
    out = (ctypes.c_int64 * 4)()
    _check(_L.gs_batch_stats(cache.handle, _stream(stream), out))
    return {"slow_refills": int(out[0]), "queued_rescans": int(out[1]), "refreshed_nodes": int(out[2]),
            "philox_blocks": int(out[3])}


def gs_cache_profile_begin(cache: Cache, max_batches: int):
    _check(_L.gs_cache_profile_begin(cache.handle, int(max_batches)))


def gs_cache_profile_end(cache: Cache, stream=None):
    """Synchronises; ({'row_counts': ms, 'scan': ms, 'finish': ms, 'relabel': ms}, batches timed)."""
    ms = (ctypes.c_double * 4)()
    nb = ctypes.c_int64()
    _check(_L.gs_cache_profile_end(cache.handle, _stream(stream), ms, ctypes.byref(nb)))
    return dict(zip(("row_counts", "scan", "finish", "relabel"), [float(x) for x in ms])), int(nb.value)


def gs_sync_status(cache: Cache, stream=None):
    _check(_L.gs_sync_status(cache.handle, _stream(stream)))


def gs_debug_set_grid_cap(max_blocks: int):
    """Process-wide test knob: cap every kernel's grid at max_blocks blocks (0 = designed grids)."""
    _check(_L.gs_debug_set_grid_cap(int(max_blocks)))


def gs_cache_set_tuning(cache: Cache, lambda_otf=0.0, lambda_full=0.0, hub_degree=0):
    _check(_L.gs_cache_set_tuning(cache.handle, float(lambda_otf), float(lambda_full), int(hub_degree)))


def gs_alu_ceiling(what: int, milliseconds: int = 20, stream=None) -> float:
    """Measured rate (units per second) of 0: Philox blocks with the threshold test, 1: wide multiplies, 2: logic ops."""
    out = ctypes.c_double()
    _check(_L.gs_alu_ceiling(int(what), int(milliseconds), _stream(stream), ctypes.byref(out)))
    return float(out.value)


def gs_cache_set_dedup(cache: Cache, method: int):
    """GS_DEDUP_DIRECT / GS_DEDUP_HASH / GS_DEDUP_SORT for the following batches on this cache."""
    _check(_L.gs_cache_set_dedup(cache.handle, int(method)))


# ---------------------------------------------------------------- training operators
# Small calls are bound by this file: addresses and streams go to the library as plain integers, and the strided
# operands of a call as one array.
_DTYPE = {torch.float32: GS_F32, torch.bfloat16: GS_BF16}
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def _addr(t):
    return None if t is None else t.data_ptr()


def _on(stream, t: torch.Tensor):
    """The stream's handle; by default the current one of the tensor's device."""
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(t.get_device()) if _raw_stream is not None else torch.cuda.current_stream(t.device).cuda_stream


def _new(shape, dtype, like: torch.Tensor, stream, rest=None) -> torch.Tensor:
    """An output that the caller did not bring: memory of the stream the call runs on, so that nothing queued on another
    stream for the memory's last owner can still write to it.  `rest`: what rows that the kernels do not write hold, where
    there may be such rows (an array at its bound, whose length only the device knows)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return _new(shape, dtype, like, None, rest)
    if rest is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    return torch.full(shape, rest, dtype=dtype, device=like.device)


def _dtype(t: torch.dtype) -> int:
    code = _DTYPE.get(t)
    if code is None:
        raise TypeError("float32 or bfloat16 expected, got %s" % t)
    return code


def _rows_2d(t: torch.Tensor, what: str) -> torch.Tensor:
    stride = t.stride()
    if len(stride) != 2 or (stride[1] != 1 and t.shape[1] > 1) or not t.is_cuda:
        raise TypeError("%s must be a row-major 2-D CUDA tensor" % what)
    return t


def _ids_1d(t: torch.Tensor, what: str) -> torch.Tensor:
    if t.dtype is not torch.int32 or not t.is_cuda or t.dim() != 1 or not t.is_contiguous():
        raise TypeError("%s must be a contiguous 1-D int32 CUDA tensor" % what)
    return t


def _counter(t: torch.Tensor, what: str):
    """Address of a device scalar (None: there is none)."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or not t.is_cuda or t.numel() < 1:
        raise TypeError("%s must be an int32 CUDA tensor of one element" % what)
    return t.data_ptr()


def _workspace(t: torch.Tensor):
    """(address, bytes) of a call's workspace."""
    if t.dtype is not torch.uint8 or not t.is_cuda or not t.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 CUDA tensor")
    return t.data_ptr(), t.numel()


def _ld(t: torch.Tensor) -> int:
    """Row pitch; a single row may carry any stride."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def gs_embedding_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out: torch.Tensor = None,
                        out_dtype: torch.dtype = None, count: torch.Tensor = None, stream=None) -> torch.Tensor:
    """out[p] = scale * table[ids[p]]; ids outside the table give rows of zeros.  `count`: a 0-d int32 CUDA tensor
    with the list's length (`ids` is then the bound; rows behind it are zeros, or left as they are in a given `out`)."""
    _rows_2d(table, "table")
    _ids_1d(ids, "ids")
    if out is None:
        out = _new((ids.numel(), table.shape[1]), out_dtype or table.dtype, table, stream, None if count is None else 0)
    else:
        _rows_2d(out, "out")
        if out.shape[0] < ids.numel() or out.shape[1] != table.shape[1]:
            raise ValueError("out must be [len(ids), dim]")
    _check(_L.gs_embedding_lookup(_addr(table), _dtype(table.dtype), table.shape[0], table.shape[1], _ld(table), _addr(ids),
                                  _counter(count, "count"), ids.numel(), float(scale), _addr(out), _dtype(out.dtype), _ld(out),
                                  _on(stream, out)))
    return out


def gs_embedding_workspace_bytes(num_ids: int, table_rows: int, dim: int) -> int:
    out = ctypes.c_size_t()
    _check(_L.gs_embedding_workspace_bytes(int(num_ids), int(table_rows), int(dim), ctypes.byref(out)))
    return out.value


def _embedding_grad_args(dout, ids):
    _rows_2d(dout, "dout")
    _ids_1d(ids, "ids")
    if dout.shape[0] < ids.numel():
        raise ValueError("dout has fewer rows than there are ids")


def gs_embedding_backward(dout: torch.Tensor, ids: torch.Tensor, table_rows: int, workspace: torch.Tensor, scale: float = 1.0,
                          out: torch.Tensor = None, out_dtype: torch.dtype = None, count: torch.Tensor = None,
                          stream=None) -> torch.Tensor:
    """Gradient of the whole table: row r = scale * sum of dout[p] over ids[p] == r, zeros elsewhere."""
    _embedding_grad_args(dout, ids)
    if out is None:
        out = _new((int(table_rows), dout.shape[1]), out_dtype or dout.dtype, dout, stream)
    else:
        _rows_2d(out, "out")
        if tuple(out.shape) != (int(table_rows), dout.shape[1]):
            raise ValueError("out must be [table_rows, dim]")
    _check(_L.gs_embedding_backward(_addr(dout), _dtype(dout.dtype), _ld(dout), _addr(ids), _counter(count, "count"), ids.numel(),
                                    int(table_rows), dout.shape[1], float(scale), _addr(out), _dtype(out.dtype), _ld(out),
                                    *_workspace(workspace), _on(stream, workspace)))
    return out


def gs_embedding_backward_sparse(dout: torch.Tensor, ids: torch.Tensor, table_rows: int, workspace: torch.Tensor,
                                 scale: float = 1.0, rows: torch.Tensor = None, num_rows: torch.Tensor = None,
                                 grad: torch.Tensor = None, out_dtype: torch.dtype = None, count: torch.Tensor = None,
                                 stream=None):
    """The rows of the gradient that occur: (ids ascending, their number as int32[1], sums); -1 / zeros behind them."""
    _embedding_grad_args(dout, ids)
    n, d = ids.numel(), dout.shape[1]
    if rows is None:
        rows = _new(n, torch.int32, dout, stream)
    if num_rows is None:
        num_rows = _new(1, torch.int32, dout, stream)
    if grad is None:
        grad = _new((n, d), out_dtype or dout.dtype, dout, stream)
    _ids_1d(rows, "rows")
    _rows_2d(grad, "grad")
    if rows.numel() < n or grad.shape[0] < n or grad.shape[1] != d:
        raise ValueError("rows / grad must hold one entry per id")
    _check(_L.gs_embedding_backward_sparse(_addr(dout), _dtype(dout.dtype), _ld(dout), _addr(ids), _counter(count, "count"), n, int(table_rows), d,
                                           float(scale), _addr(rows), _counter(num_rows, "num_rows"), _addr(grad), _dtype(grad.dtype), _ld(grad),
                                           *_workspace(workspace), _on(stream, workspace)))
    return rows, num_rows, grad


def _csr_block(indptr, indices, num_src, counts):
    _ids_1d(indptr, "indptr")
    _ids_1d(indices, "indices")
    nd, ns, ne = (None, None, None) if counts is None else (_counter(c, "each of counts") for c in counts)
    return _CBlock(indptr.numel() - 1, int(num_src), indices.numel(), nd, ns, ne, indptr.data_ptr(), indices.data_ptr())


def _heads(dtype, *operands):
    """gs_heads of (tensor, name, rows, heads, head_dim), one behind the other; returns (array, addresses)."""
    words = []
    for t, what, rows, heads, dim in operands:
        shape, stride = t.shape, t.stride()
        if t.dtype is not dtype or len(shape) != 3 or shape[0] < rows or shape[1] != heads or shape[2] != dim or not t.is_cuda or \
                (stride[2] != 1 and dim > 1):
            raise TypeError("%s must be a CUDA tensor [%d, %d, %d] of %s with a contiguous last dimension" % (what, rows, heads, dim, dtype))
        words += (t.data_ptr(), stride[0] if shape[0] > 1 else max(stride[0], dim), stride[1] if heads > 1 else dim)
    words = array("q", words)
    at = words.buffer_info()[0]
    return words, [at + 24 * i for i in range(len(operands))]


def gs_block_attention_workspace_bytes(num_dst: int, num_src: int, num_edges: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    """Bytes for gs_block_attention_forward, gs_block_reverse and gs_block_attention_backward on such a block."""
    out = ctypes.c_size_t()
    _check(_L.gs_block_attention_workspace_bytes(int(num_dst), int(num_edges), int(q_heads), int(head_dim), ctypes.byref(out)))
    return out.value


def gs_block_attention_forward(indptr: torch.Tensor, indices: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                               workspace: torch.Tensor, scale: float = None, max_row: int = 0, out: torch.Tensor = None,
                               lse: torch.Tensor = None, counts=None, stream=None):
    """Attention of a block's destinations (q: [dst, q_heads, head_dim]) over their sources (k, v: [src, kv_heads,
    head_dim]); indptr, indices: the block's int32 arrays; an index outside [0, src) is masked.  `scale` defaults to
    1 / sqrt(head_dim); `max_row`: an upper bound on a row's edges (the fan-out) if one is known; `counts`: the
    device scalars of Block.counts_device() when the arrays are only bounds.  Returns (out, lse); rows of q that the block
    does not have get zeros and -inf, or are left as they are in given arrays."""
    n, hq, d = q.shape
    hk = k.shape[1]
    if indptr.numel() - 1 > n:
        raise ValueError("q has fewer rows than the block has destinations")
    b = _csr_block(indptr, indices, k.shape[0], counts)
    exact = counts is None and n == b.max_dst
    if out is None:
        out = _new((n, hq, d), q.dtype, q, stream, None if exact else 0)
    if lse is None:
        lse = _new((n, hq), torch.float32, q, stream, None if exact else -math.inf)
    elif lse.dtype != torch.float32 or not lse.is_cuda or not lse.is_contiguous() or lse.shape[0] < b.max_dst or lse.shape[1] != hq:
        raise TypeError("lse must be a contiguous float32 tensor [dst, q_heads]")
    keep, (pq, pk, pv, po) = _heads(q.dtype, (q, "q", b.max_dst, hq, d), (k, "k", b.max_src, hk, d), (v, "v", b.max_src, hk, d),
                                    (out, "out", b.max_dst, hq, d))
    _check(_L.gs_block_attention_forward(ctypes.byref(b), int(max_row), _dtype(q.dtype), hq, hk, d,
                                         d ** -0.5 if scale is None else float(scale), pq, pk, pv, po, _addr(lse), *_workspace(workspace), _on(stream, workspace)))
    return out, lse


def gs_block_reverse(indptr: torch.Tensor, indices: torch.Tensor, num_src: int, workspace: torch.Tensor, rev_indptr: torch.Tensor = None,
                     rev_dst: torch.Tensor = None, rev_edge: torch.Tensor = None, counts=None, stream=None):
    """The block in source order: (int32[num_src + 1] offsets, int32[edges] destinations, int32[edges] edges they came
    from), masked edges left out."""
    b = _csr_block(indptr, indices, num_src, counts)
    if rev_indptr is None:
        rev_indptr = _new(b.max_src + 1, torch.int32, indptr, stream)
    if rev_dst is None:
        rev_dst = _new(b.max_edges, torch.int32, indptr, stream)
    if rev_edge is None:
        rev_edge = _new(b.max_edges, torch.int32, indptr, stream)
    if _ids_1d(rev_indptr, "rev_indptr").numel() < b.max_src + 1 or _ids_1d(rev_dst, "rev_dst").numel() < b.max_edges or \
            _ids_1d(rev_edge, "rev_edge").numel() < b.max_edges:
        raise ValueError("rev_indptr / rev_dst / rev_edge are too small")
    _check(_L.gs_block_reverse(ctypes.byref(b), _addr(rev_indptr), _addr(rev_dst), _addr(rev_edge), *_workspace(workspace), _on(stream, workspace)))
    return rev_indptr, rev_dst, rev_edge


def gs_block_attention_backward(indptr: torch.Tensor, indices: torch.Tensor, reverse, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                                out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor, workspace: torch.Tensor, scale: float = None,
                                max_row: int = 0, dq: torch.Tensor = None, dk: torch.Tensor = None, dv: torch.Tensor = None, counts=None,
                                stream=None):
    """Gradients of gs_block_attention_forward; `reverse` is what gs_block_reverse returned.  Returns (dq, dk, dv); rows that
    the block does not have get zeros, or are left as they are in given arrays."""
    n, hq, d = q.shape
    hk = k.shape[1]
    b = _csr_block(indptr, indices, k.shape[0], counts)
    rev_indptr, rev_dst, rev_edge = reverse
    if _ids_1d(rev_indptr, "rev_indptr").numel() < b.max_src + 1 or _ids_1d(rev_dst, "rev_dst").numel() < b.max_edges or \
            _ids_1d(rev_edge, "rev_edge").numel() < b.max_edges:
        raise ValueError("reverse belongs to another block")
    if lse.dtype != torch.float32 or not lse.is_cuda or not lse.is_contiguous() or lse.shape[0] < b.max_dst or lse.shape[1] != hq:
        raise TypeError("lse must be a contiguous float32 tensor [dst, q_heads]")
    rest = lambda rows, bound: None if counts is None and rows == bound else 0  # noqa: E731
    dq = _new((n, hq, d), q.dtype, q, stream, rest(n, b.max_dst)) if dq is None else dq
    dk = _new((k.shape[0], hk, d), q.dtype, q, stream, rest(k.shape[0], b.max_src)) if dk is None else dk
    dv = _new((v.shape[0], hk, d), q.dtype, q, stream, rest(v.shape[0], b.max_src)) if dv is None else dv
    t = q.dtype
    keep, (pq, pk, pv, po, pdo, pdq, pdk, pdv) = _heads(
        t, (q, "q", b.max_dst, hq, d), (k, "k", b.max_src, hk, d), (v, "v", b.max_src, hk, d), (out, "out", b.max_dst, hq, d),
        (dout, "dout", b.max_dst, hq, d), (dq, "dq", b.max_dst, hq, d), (dk, "dk", b.max_src, hk, d), (dv, "dv", b.max_src, hk, d))
    _check(_L.gs_block_attention_backward(ctypes.byref(b), int(max_row), _addr(rev_indptr), _addr(rev_dst), _addr(rev_edge), _dtype(t), hq, hk, d,
                                          d ** -0.5 if scale is None else float(scale), pq, pk, pv, po, _addr(lse), pdo, pdq, pdk, pdv,
                                          *_workspace(workspace), _on(stream, workspace)))
    return dq, dk, dv


def gs_xent_workspace_bytes(rows: int, vocab: int, dim: int, dtype: torch.dtype = torch.bfloat16) -> int:
    out = ctypes.c_size_t()
    _check(_L.gs_xent_workspace_bytes(int(rows), int(vocab), int(dim), _dtype(dtype), ctypes.byref(out)))
    return out.value


def _xent_args(hidden, table, labels):
    _rows_2d(hidden, "hidden")
    _rows_2d(table, "table")
    _ids_1d(labels, "labels")
    if hidden.dtype != table.dtype or hidden.shape[1] != table.shape[1]:
        raise TypeError("hidden and table must have one dtype and one width")
    if labels.numel() != hidden.shape[0]:
        raise ValueError("one label per hidden row expected")


def _f32_rows(t, what, n):
    if t.dtype != torch.float32 or not t.is_cuda or t.dim() != 1 or not t.is_contiguous() or t.numel() < n:
        raise TypeError("%s must be a contiguous float32 CUDA tensor with one entry per row" % what)
    return t


def gs_xent_forward(hidden: torch.Tensor, table: torch.Tensor, labels: torch.Tensor, workspace: torch.Tensor, scale: float = 1.0,
                    loss: torch.Tensor = None, lse: torch.Tensor = None, stream=None):
    """loss[n] = lse[n] - scale <hidden[n], table[labels[n]]>, lse over all rows of the table; labels outside it: loss 0."""
    _xent_args(hidden, table, labels)
    n = hidden.shape[0]
    loss = _new(n, torch.float32, hidden, stream) if loss is None else _f32_rows(loss, "loss", n)
    lse = _new(n, torch.float32, hidden, stream) if lse is None else _f32_rows(lse, "lse", n)
    _check(_L.gs_xent_forward(_addr(hidden), _ld(hidden), _addr(table), _ld(table), _dtype(hidden.dtype), n, table.shape[0], hidden.shape[1],
                              float(scale), _addr(labels), _addr(loss), _addr(lse), *_workspace(workspace), _on(stream, workspace)))
    return loss, lse


def gs_xent_backward(hidden: torch.Tensor, table: torch.Tensor, labels: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor,
                     workspace: torch.Tensor, scale: float = 1.0, dhidden: torch.Tensor = None, dtable: torch.Tensor = None,
                     out_dtype: torch.dtype = None, stream=None):
    """Gradients of gs_xent_forward for the upstream gradient dloss (float32, one per row).  Returns (dhidden, dtable)."""
    _xent_args(hidden, table, labels)
    n, d = hidden.shape
    _f32_rows(lse, "lse", n)
    _f32_rows(dloss, "dloss", n)
    t = out_dtype or hidden.dtype
    dhidden = _new((n, d), t, hidden, stream) if dhidden is None else _rows_2d(dhidden, "dhidden")
    dtable = _new(tuple(table.shape), dhidden.dtype, hidden, stream) if dtable is None else _rows_2d(dtable, "dtable")
    if tuple(dhidden.shape) != (n, d) or dtable.shape != table.shape or dhidden.dtype != dtable.dtype:
        raise ValueError("dhidden / dtable must have the shapes of hidden / table and one dtype")
    _check(_L.gs_xent_backward(_addr(hidden), _ld(hidden), _addr(table), _ld(table), _dtype(hidden.dtype), n, table.shape[0], d, float(scale),
                               _addr(labels), _addr(lse), _addr(dloss), _addr(dhidden), _ld(dhidden), _addr(dtable), _ld(dtable),
                               _dtype(dhidden.dtype), *_workspace(workspace), _on(stream, workspace)))
    return dhidden, dtable


def gs_train_status(stream=None):
    """Synchronises; raises if a kernel of the training operators ever gave up waiting, and so left results partly unwritten:
    call it before they are kept."""
    _check(_L.gs_train_status((torch.cuda.current_stream() if stream is None else stream).cuda_stream))


# ---------------------------------------------------------------- around an attention layer: norms, rows in 8 bits, gradient clipping
def _one_device(*tensors):
    """All operands of a call are memory of one GPU: the call's."""
    device = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("the operands are on different devices")
    return device


_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _run(device, fn, *args):
    """The call, on the operands' device."""
    if device == _current_device():
        status = fn(*args)
    else:
        with torch.cuda.device(device):
            status = fn(*args)
    if status != 0:
        _check(status)


def _new_like(t: torch.Tensor, stream, rest=None) -> torch.Tensor:
    """An output of the shape and dtype of a contiguous tensor, or of a row-major one with a pitch (see _new); without its
    arguments to parse an allocation takes half the time."""
    if stream is None and rest is None:
        return torch.empty_like(t)
    return _new(tuple(t.shape), t.dtype, t, stream, rest)


def _norm_rows(t, what, like):
    stride = t.stride()
    if len(stride) != 2 or (stride[1] != 1 and t.shape[1] > 1) or not t.is_cuda or t.dtype is not like.dtype or t.shape != like.shape:
        _rows_2d(t, what)
        raise TypeError("%s must have the dtype and shape of the normalised rows" % what)
    return t


def _norm_weight(weight, dim):
    if weight is None:
        return None, GS_F32
    if weight.shape != (dim,) or not weight.is_cuda or not weight.is_contiguous():
        raise TypeError("weight must be a contiguous CUDA tensor [%d]" % dim)
    return weight.data_ptr(), _dtype(weight.dtype)


def _opt(t):
    """(address, row pitch) of an operand that may be missing."""
    return (None, 0) if t is None else (t.data_ptr(), _ld(t))


def gs_rms_norm_workspace_bytes(rows: int, dim: int) -> int:
    """Bytes for gs_rms_norm_backward of so many rows."""
    out = ctypes.c_size_t()
    _check(_L.gs_rms_norm_workspace_bytes(int(rows), int(dim), ctypes.byref(out)))
    return out.value


def _norm_inputs(x, weight, residual, hidden, stream, count):
    _rows_2d(x, "x")
    if residual is not None:
        _norm_rows(residual, "residual", x)
        hidden = _new_like(x, stream, None if count is None else 0) if hidden is None else _norm_rows(hidden, "hidden", x)
    elif hidden is not None:
        _norm_rows(hidden, "hidden", x)
    return hidden, _norm_weight(weight, x.shape[1])


def gs_rms_norm_forward(x: torch.Tensor, weight: torch.Tensor = None, residual: torch.Tensor = None, eps: float = 1e-6, out: torch.Tensor = None,
                        hidden: torch.Tensor = None, count: torch.Tensor = None, stream=None):
    """h = x + residual; out = weight * h / sqrt(mean(h^2) + eps), row by row.  Returns (out, h); h is x itself without a residual.
    `hidden` (h) and `out` may each be x or residual, but not both the same.  `count`: a 0-d int32 CUDA tensor with the number of rows (x is then the
    bound; rows behind it are zeros, or left as they are in given arrays)."""
    hidden, (w, wt) = _norm_inputs(x, weight, residual, hidden, stream, count)
    out = _new_like(x, stream, None if count is None else 0) if out is None else _norm_rows(out, "out", x)
    device = _one_device(x, weight, residual, hidden, out, count)
    rows, dim = x.shape
    _run(device, _L.gs_rms_norm_forward, x.data_ptr(), _ld(x), *_opt(residual), _dtype(x.dtype), w, wt, _counter(count, "count"), rows, dim, float(eps),
         *_opt(hidden), out.data_ptr(), _ld(out), _on(stream, x))
    return out, x if hidden is None else hidden


def gs_rms_norm_coded(x: torch.Tensor, out: "CodedRows", weight: torch.Tensor = None, residual: torch.Tensor = None, eps: float = 1e-6,
                      hidden: torch.Tensor = None, count: torch.Tensor = None, stream=None):
    """gs_rms_norm_forward with the result in 8 bits: row p of `out` (a store with block 1 and heads * head_dim = dim).  Returns (out, h)."""
    hidden, (w, wt) = _norm_inputs(x, weight, residual, hidden, stream, count)
    device = _one_device(x, weight, residual, hidden, out.codes, count)
    rows, dim = x.shape
    _run(device, _L.gs_rms_norm_coded, x.data_ptr(), _ld(x), *_opt(residual), _dtype(x.dtype), w, wt, _counter(count, "count"), rows, dim, float(eps),
         *_opt(hidden), out.address, _on(stream, x))
    return out, x if hidden is None else hidden


def gs_rms_norm_backward(hidden: torch.Tensor, dout: torch.Tensor, workspace: torch.Tensor, weight: torch.Tensor = None, dhidden: torch.Tensor = None,
                         eps: float = 1e-6, dx: torch.Tensor = None, dweight: torch.Tensor = None, count: torch.Tensor = None, stream=None):
    """Gradients of gs_rms_norm_forward for what it normalised.  `dhidden`: the gradient that arrives at h itself.  Returns (dx,
    dweight); dx is the residual's gradient too, dweight None without a weight.  `dx` may be hidden, dhidden or dout."""
    _rows_2d(hidden, "hidden")
    _norm_rows(dout, "dout", hidden)
    if dhidden is not None:
        _norm_rows(dhidden, "dhidden", hidden)
    w, wt = _norm_weight(weight, hidden.shape[1])
    dx = _new_like(hidden, stream, None if count is None else 0) if dx is None else _norm_rows(dx, "dx", hidden)
    if weight is None:
        if dweight is not None:
            raise ValueError("there is no weight")
    elif dweight is None:
        dweight = _new_like(weight, stream)
    elif dweight.dtype is not weight.dtype or _norm_weight(dweight, hidden.shape[1])[0] is None:
        raise TypeError("dweight must have the dtype of weight")
    device = _one_device(hidden, dout, workspace, weight, dhidden, dx, dweight, count)
    rows, dim = hidden.shape
    _run(device, _L.gs_rms_norm_backward, hidden.data_ptr(), _ld(hidden), dout.data_ptr(), _ld(dout), *_opt(dhidden), _dtype(hidden.dtype), w, wt, _counter(count, "count"),
         rows, dim, float(eps), dx.data_ptr(), _ld(dx), _addr(dweight), *_workspace(workspace), _on(stream, workspace))
    return dx, dweight


class _CCoded(ctypes.Structure):
    _fields_ = [("d_codes", ctypes.c_void_p), ("d_scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("scale_stride", ctypes.c_int64), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32)]


class CodedRows:
    """Rows in 8 bits over two caller-owned tensors (see gs_coded in include/gs.h): codes [rows, heads, pitch] (float8_e4m3fn or
    uint8; pitch = head_dim rounded up to 16) and scales uint8 [ceil(rows / block), heads].  Tensors of zeros are a store of zero
    rows.  A store holds an int32 per row and two per block beside them, for writes by id; two of those on one store may not overlap.
    Making a store waits until these are set, so that writes on any stream find them; their memory is not given back while a write that
    was queued before the store went is still under way.  Codes and scales are tensors like any other in this; a graph that holds a
    write needs the store to live as long as it is replayed."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, head_dim: int, block: int = 1):
        head_dim, block = int(head_dim), int(block)
        if block < 1 or block > 64 or block & (block - 1):
            raise ValueError("block must be a power of two from 1 to 64")
        pitch = (head_dim + 15) // 16 * 16
        if codes.dtype not in (torch.float8_e4m3fn, torch.uint8) or not codes.is_cuda or codes.dim() != 3 or head_dim < 1 or codes.shape[2] != pitch or \
                codes.stride(2) != 1 or (codes.shape[1] > 1 and codes.stride(1) != pitch):
            raise TypeError("codes must be a CUDA tensor [rows, heads, %d] of float8_e4m3fn or uint8, heads one behind the other" % pitch)
        rows, heads = codes.shape[0], codes.shape[1]
        if scales.dtype != torch.uint8 or tuple(scales.shape) != ((rows + block - 1) // block, heads) or (heads > 1 and scales.stride(1) != 1):
            raise TypeError("scales must be a uint8 tensor [ceil(rows / block), heads]")
        device = _one_device(codes, scales)
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a store cannot be made while a graph is captured")
        claims = torch.full((rows + (2 * scales.shape[0] + 2 if block > 1 else 0),), -1, dtype=torch.int32, device=torch.device("cuda", device))
        made_on = torch.cuda.current_stream(device)
        made_on.synchronize()
        self._made_on = made_on.cuda_stream
        self._set(codes, scales, head_dim, block, claims)

    def _set(self, codes, scales, head_dim, block, claims):
        self.codes, self.scales, self.claims = codes, scales, claims
        self.rows, self.num_heads, self.head_dim, self.block = codes.shape[0], codes.shape[1], head_dim, block
        stride = codes.stride(0) if self.rows > 1 else self.num_heads * codes.shape[2]
        self._c = _CCoded(codes.data_ptr(), scales.data_ptr(), self.rows, stride, scales.stride(0) if scales.shape[0] > 1 else self.num_heads,
                          self.num_heads, head_dim, block)
        self.address = ctypes.addressof(self._c)

    def heads(self, first: int, end: int) -> "CodedRows":
        """The heads [first, end) as a store over the same memory (keys and values of one cache, say)."""
        if not 0 <= first < end <= self.num_heads:
            raise ValueError("heads [%d, %d) of %d" % (first, end, self.num_heads))
        part = object.__new__(CodedRows)
        part._made_on = self._made_on
        part._set(self.codes[:, first:end], self.scales[:, first:end], self.head_dim, self.block, self.claims)
        return part


def gs_coded_rows(rows: int, heads: int, head_dim: int, block: int = 16, device=None) -> CodedRows:
    """A store of `rows` zero rows."""
    device = torch.device("cuda") if device is None else device
    codes = torch.zeros((int(rows), int(heads), (int(head_dim) + 15) // 16 * 16), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
    return CodedRows(codes, torch.zeros(((int(rows) + int(block) - 1) // int(block), int(heads)), dtype=torch.uint8, device=device), head_dim, block)


def gs_coded_write(to: CodedRows, rows: torch.Tensor, ids: torch.Tensor = None, first: int = 0, count: torch.Tensor = None, stream=None) -> CodedRows:
    """rows[p] ([n, heads, head_dim], float32 or bfloat16) into row ids[p] of the store, or first + p.  Ids outside the store are
    skipped, of equal ids the last counts.  `count`: the device's number of rows (n is then the bound)."""
    n = rows.shape[0] if ids is None else _ids_1d(ids, "ids").numel()
    keep, (p,) = _heads(rows.dtype, (rows, "rows", n, to.num_heads, to.head_dim))
    device = _one_device(to.codes, rows, ids, count)
    handle = _on(stream, to.codes)
    if ids is not None and handle != to._made_on:            # the caller does not see the claims, and cannot guard their memory
        to.claims.record_stream(torch.cuda.current_stream(device) if stream is None else stream)
    _run(device, _L.gs_coded_write, to.address, _dtype(rows.dtype), p, _addr(ids), int(first), _counter(count, "count"), n, _addr(to.claims), handle)
    return to


def gs_coded_read(store: CodedRows, ids: torch.Tensor = None, first: int = 0, num_rows: int = None, out: torch.Tensor = None,
                  out_dtype: torch.dtype = torch.bfloat16, count: torch.Tensor = None, stream=None) -> torch.Tensor:
    """out[p] = row ids[p] of the store, or first + p for p < num_rows (default: to its end); ids outside it give zeros."""
    n = _ids_1d(ids, "ids").numel() if ids is not None else (store.rows - int(first) if num_rows is None else int(num_rows))
    if n < 0:
        raise ValueError("no rows from %d on" % first)
    if out is None:
        out = _new((n, store.num_heads, store.head_dim), out_dtype, store.codes, stream, None if count is None else 0)
    keep, (p,) = _heads(out.dtype, (out, "out", n, store.num_heads, store.head_dim))
    device = _one_device(store.codes, ids, out, count)
    _run(device, _L.gs_coded_read, store.address, _addr(ids), int(first), _counter(count, "count"), n, _dtype(out.dtype), p, _on(stream, store.codes))
    return out


def gs_coded_attention_workspace_bytes(num_dst: int, num_edges: int, q_heads: int, head_dim: int) -> int:
    """Bytes for gs_coded_attention_forward on such a block."""
    out = ctypes.c_size_t()
    _check(_L.gs_coded_attention_workspace_bytes(int(num_edges), int(q_heads), int(head_dim), ctypes.byref(out)))
    return out.value


def gs_coded_attention_forward(indptr: torch.Tensor, indices: torch.Tensor, q: torch.Tensor, k: CodedRows, v: CodedRows, workspace: torch.Tensor,
                               rows: torch.Tensor = None, scale: float = None, max_row: int = 0, out: torch.Tensor = None, lse: torch.Tensor = None,
                               counts=None, stream=None):
    """gs_block_attention_forward with keys and values in 8 bits (k, v: stores, or parts of one).  `rows`: the store's row of every
    source of the block (its input nodes, say); without it a source is its row.  Returns (out, lse)."""
    n, hq, d = q.shape
    if indptr.numel() - 1 > n:
        raise ValueError("q has fewer rows than the block has destinations")
    b = _csr_block(indptr, indices, k.rows if rows is None else _ids_1d(rows, "rows").numel(), counts)
    exact = counts is None and n == b.max_dst
    if out is None:
        out = _new_like(q, stream) if exact and q.is_contiguous() else _new((n, hq, d), q.dtype, q, stream, None if exact else 0)
    if lse is None:
        lse = _new((n, hq), torch.float32, q, stream, None if exact else -math.inf)
    elif lse.dtype != torch.float32 or not lse.is_cuda or not lse.is_contiguous() or lse.dim() != 2 or lse.shape[0] < b.max_dst or lse.shape[1] != hq:
        raise TypeError("lse must be a contiguous float32 tensor [dst, q_heads]")
    keep, (pq, po) = _heads(q.dtype, (q, "q", b.max_dst, hq, d), (out, "out", b.max_dst, hq, d))
    device = _one_device(q, indptr, indices, k.codes, v.codes, workspace, rows, out, lse, *(() if counts is None else counts))
    _run(device, _L.gs_coded_attention_forward, ctypes.byref(b), _addr(rows), int(max_row), _dtype(q.dtype), hq, d, d ** -0.5 if scale is None else float(scale),
         pq, k.address, v.address, po, _addr(lse), *_workspace(workspace), _on(stream, workspace))
    return out, lse


def _dense(t: torch.Tensor, what: str) -> torch.Tensor:
    """A tensor whose elements fill its memory without gaps, in any order of dimensions."""
    if not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % what)
    if not t.is_contiguous():
        at = 1
        for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
            if stride != at:
                raise TypeError("%s has gaps or overlaps in memory" % what)
            at *= size
    return t


def gs_grad_workspace_bytes(num_grads: int) -> int:
    out = ctypes.c_size_t()
    _check(_L.gs_grad_workspace_bytes(int(num_grads), ctypes.byref(out)))
    return out.value


def _grad_list(grads, out, counts):
    """gs_grad of every gradient, six words each."""
    if out is not None and len(out) != len(grads) or counts is not None and len(counts) != len(grads):
        raise ValueError("one result and one count per gradient expected")
    words = []
    for i, g in enumerate(grads):
        if not (g.is_cuda and g.is_contiguous()):
            _dense(g, "each gradient")
        n, p, rows, row_elems = g.numel(), g.data_ptr(), 0, 0
        o = p
        if out is not None and out[i] is not g:
            x = out[i]
            if x.dtype is not g.dtype or x.shape != g.shape or x.stride() != g.stride() or not x.is_cuda:
                raise TypeError("a result must have the dtype, shape and strides of its gradient")
            o = x.data_ptr()
        if counts is not None and counts[i] is not None:
            if g.dim() < 1 or not g.is_contiguous():
                raise TypeError("a gradient with a count must be a contiguous tensor of rows")
            rows, row_elems = _counter(counts[i], "each of counts"), n // g.shape[0] if n else 0
        words += (p, o, n, rows, row_elems, _dtype(g.dtype))
    return array("q", words or (0,))


def gs_grad_norm(grads, workspace: torch.Tensor, norm: torch.Tensor = None, counts=None, stream=None) -> torch.Tensor:
    """The norm over all numbers of a list of gradients, as float32[1] on the device.  `counts`: for each gradient None, or the
    device's number of its rows that count (as gs_embedding_backward_sparse returns it)."""
    grads = list(grads)
    norm = _new(1, torch.float32, workspace, stream) if norm is None else _f32_rows(norm, "norm", 1)
    device = _one_device(workspace, norm, *grads, *(counts or ()))
    words = _grad_list(grads, None, counts)
    _run(device, _L.gs_grad_norm, words.buffer_info()[0], len(grads), _addr(norm), *_workspace(workspace), _on(stream, workspace))
    return norm


def gs_grad_clip(grads, max_norm: float, workspace: torch.Tensor, out=None, norm: torch.Tensor = None, counts=None, stream=None) -> torch.Tensor:
    """Scales a list of gradients by min(1, max_norm / (norm + 1e-6)), in place or into the list `out`, and returns their norm before
    that.  `counts`: as for gs_grad_norm; rows behind a count are left as they are.  Nothing waits for the device."""
    grads = list(grads)
    norm = _new(1, torch.float32, workspace, stream) if norm is None else _f32_rows(norm, "norm", 1)
    device = _one_device(workspace, norm, *grads, *(out or ()), *(counts or ()))
    words = _grad_list(grads, out, counts)
    _run(device, _L.gs_grad_clip, words.buffer_info()[0], len(grads), float(max_norm), _addr(norm), *_workspace(workspace), _on(stream, workspace))
    return norm
