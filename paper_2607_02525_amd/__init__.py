"""Python binding of libpeek (include/peek.h): batched longest-prefix match of
a waiting queue against a KV prefix-cache radix tree, plus the queue signals
(prefix-sharing clusters and per-cache-node pending demand), and attention over
the cache's 8-bit pages, on MI355X.

Argument marshalling only: every step runs in the library's HIP kernels.
Device arrays are torch tensors on the current HIP device (torch is used for
device memory and streams); host arrays are numpy. Each function has the
name of the C entry point it calls and raises PeekError on failure. There is
no CPU fallback: importing this module fails if libpeek.so is not built.
"""
from __future__ import annotations

import ctypes
import math
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpeek.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run `python paper_2607_02525_amd/build.py` "
                      "(or __graft_entry__.build()) first")

# torch's HIP runtime goes in first: libpeek.so then binds to that same
# libamdhip64.so.7 (same soname) instead of loading the system copy beside
# it. Two HIP runtimes in one process do not share the device: the second
# to initialise reports no device.
import torch  # noqa: E402,F401

_lib = ctypes.CDLL(LIB_PATH)

PEEK_OK = 0
PEEK_ERR_INVALID_ARGUMENT = -1
PEEK_ERR_INVALID_TREE = -2
PEEK_ERR_OUT_OF_MEMORY = -3
PEEK_ERR_DEVICE = -4
PEEK_ERR_WORKSPACE_TOO_SMALL = -5
PEEK_ERR_UNSUPPORTED_DEVICE = -6

_i32p = ctypes.POINTER(ctypes.c_int32)
_i64p = ctypes.POINTER(ctypes.c_int64)
_vp = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64

# (name, restype, argtypes) of every exported symbol in include/peek.h
EXPORTS = [
    ("peek_abi_version", ctypes.c_int32, []),
    ("peek_last_error", ctypes.c_char_p, []),
    ("peek_tree_canonical_ids", ctypes.c_int, [ctypes.c_int32, _i32p, _i64p, _i32p, _i32p]),
    ("peek_tree_from_sequences", ctypes.c_int,
     [_i32p, _i64p, ctypes.c_int64, _i32p, ctypes.POINTER(_i32p), ctypes.POINTER(_i64p), ctypes.POINTER(_i32p)]),
    ("peek_free_host", None, [_vp]),
    ("peek_cache_build", ctypes.c_int, [ctypes.c_int32, _i32p, _i64p, _i32p, _vp, ctypes.POINTER(_vp), _i32p]),
    ("peek_cache_stats", ctypes.c_int, [_vp, _i64p, _i64p, _i32p, _i64p, _i64p]),
    ("peek_cache_export", ctypes.c_int, [_vp, _i32p, _i32p, _i32p, _i32p]),
    ("peek_cache_free", ctypes.c_int, [_vp]),
    ("peek_lpm_batch", ctypes.c_int, [_vp, ctypes.c_int32, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp]),
    ("peek_queue_signals_workspace", ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int64]),
    ("peek_queue_signals", ctypes.c_int,
     [_vp, ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    ("peek_queue_signals_noalloc", ctypes.c_int,
     [_vp, ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp]),
    ("peek_evict_rank_workspace", ctypes.c_size_t, [ctypes.c_int64]),
    ("peek_evict_rank", ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    ("peek_clpm_signals", ctypes.c_int,
     [_vp, ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp, _vp, _vp,
      _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    ("peek_block_table_build", ctypes.c_int,
     [ctypes.c_int32, _i32p, _i64p, _i32p, ctypes.c_int32, _vp, ctypes.POINTER(_vp)]),
    ("peek_block_table_stats", ctypes.c_int, [_vp, _i64p, _i64p, _i32p]),
    ("peek_block_table_free", ctypes.c_int, [_vp]),
    ("peek_block_lpm_batch", ctypes.c_int, [_vp, ctypes.c_int32, _vp, _vp, _vp, _vp]),
    ("peek_offline_order_workspace", ctypes.c_size_t, [ctypes.c_int32]),
    ("peek_offline_order", ctypes.c_int,
     [ctypes.c_int32, _vp, _vp, ctypes.c_int32, _vp, _vp, ctypes.c_size_t, _vp]),
    ("peek_kv_append", ctypes.c_int,
     [_vp, _i32, _i64, _i32, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _i32, _i64, _vp]),
    ("peek_prefill_attention_workspace", ctypes.c_size_t, [_i32, _i64, _i32, _i32, _i32, _i64]),
    ("peek_prefill_attention", ctypes.c_int,
     [_vp, _i32, _i64, _i32, _i32, _i32, _i32, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _i32,
      _i64, ctypes.c_float, _vp, _i64, _i64, _vp, _vp, ctypes.c_size_t, _vp]),
    ("peek_decode_attention_workspace", ctypes.c_size_t, [_vp, _i32, _i32, _i32, _i32]),
    ("peek_decode_attention", ctypes.c_int,
     [_vp, _i32, _i32, _i32, _vp, _i64, _i64, _vp, _vp, _i32, _i64, ctypes.c_float, _vp, _i64, _i64, _vp, _vp, _vp,
      _vp, ctypes.c_size_t, _vp]),
    ("peek_kv_evict_workspace", ctypes.c_size_t, [_i32, _i32, _i32]),
    ("peek_kv_evict", ctypes.c_int,
     [_i32, _i32, _i32, _vp, _vp, _i32, _i64, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t,
      _vp]),
    ("peek_rotate_append", ctypes.c_int,
     [_vp, _i32, _i64, _i32, _i32, _i32, _i32, _vp, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp,
      _i32, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp]),
    ("peek_rotary_frequencies", ctypes.c_int,
     [_i32, ctypes.c_double, _i32, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double,
      ctypes.POINTER(ctypes.c_double)]),
    ("peek_kv_read", ctypes.c_int,
     [_vp, _i32, _i64, _i32, _vp, _vp, _vp, _i32, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp]),
    ("peek_shared_decode_attention_workspace", ctypes.c_size_t, [_vp, _i32, _i32, _i32, _i32]),
    ("peek_shared_decode_attention", ctypes.c_int,
     [_vp, _i32, _i32, _i32, _vp, _i64, _i64, _vp, _vp, _i32, _i64, _i32, _vp, _vp, _vp, ctypes.c_float, _vp, _i64,
      _i64, _vp, _vp, ctypes.c_size_t, _vp]),
    ("peek_kv_bounds", ctypes.c_int, [_vp, _i32, _vp, _vp, _vp, _i32, _i64, _vp, _vp]),
    ("peek_block_select_workspace", ctypes.c_size_t, [_vp, _i32, _i32]),
    ("peek_block_select", ctypes.c_int,
     [_vp, _vp, _i32, _i32, _i32, _vp, _i64, _i64, _vp, _vp, _i32, _i64, _i32, _i32, _i32, _vp, _vp, _vp,
      ctypes.c_size_t, _vp]),
    ("peek_sparse_decode_attention_workspace", ctypes.c_size_t, [_vp, _i32, _i32, _i32]),
    ("peek_sparse_decode_attention", ctypes.c_int,
     [_vp, _i32, _i32, _i32, _vp, _i64, _i64, _vp, _vp, _i32, ctypes.c_float, _vp, _i64, _i64, _vp, _vp,
      ctypes.c_size_t, _vp]),
]

for _name, _res, _args in EXPORTS:
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args


class PeekError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"peek status {status}: {message}")
        self.status = status


def peek_last_error() -> str:
    return (_lib.peek_last_error() or b"").decode()


def peek_abi_version() -> int:
    return int(_lib.peek_abi_version())


def _check(status: int):
    if status != PEEK_OK:
        raise PeekError(status, peek_last_error())


def _np32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def _np64(a):
    return np.ascontiguousarray(a, dtype=np.int64)


def _arg(t, name: str, dtype=None, count: int | None = None):
    """Device pointer of `t` (or None) after checking what the C entry points
    cannot: element type, contiguity, at least `count` elements, and that it
    lives on a GPU."""
    if t is None:
        return None
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if count is not None and t.numel() < count:
        raise ValueError(f"{name} needs at least {count} elements, has {t.numel()}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return t.data_ptr()


def _row_arg(t, name: str, dtype, n: int, *row: int):
    """As _arg, of n rows that are each [*row]: rows of another shape would be read and written at the wrong places.
    More rows are taken, as are the same elements in other numbers of dimensions."""
    if t is None:
        return None
    if t.shape == (n, *row):
        return _arg(t, name, dtype)
    each = math.prod(row)
    if t.dim() > 1:
        if t.dim() == 1 + len(row):
            fits = tuple(t.shape[1:]) == row and t.shape[0] >= n
        else:
            fits = t.numel() == n * each or (math.prod(t.shape[1:]) == each and t.shape[0] >= n)
        if not fits:
            raise ValueError(f"{name} must be {[n, *row]}, got {list(t.shape)}")
    return _arg(t, name, dtype, n * each)


def _queue_n(offsets) -> int:
    import torch
    if offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 1:
        raise TypeError("offsets must be a 1-D int64 tensor of n + 1 entries")
    return int(offsets.shape[0]) - 1


def _num_nodes(cache) -> int:
    if cache is None:
        return 0
    if getattr(cache, "_num_nodes", None) is None:
        cache._num_nodes = peek_cache_stats(cache)["num_nodes"]
    return cache._num_nodes


# The current stream's handle without a Stream object around it, where this torch has that (3 us less a call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def peek_tree_canonical_ids(parent, edge_offsets, edge_tokens) -> np.ndarray:
    parent, edge_offsets, edge_tokens = _np32(parent), _np64(edge_offsets), _np32(edge_tokens)
    out = np.empty(len(parent), dtype=np.int32)
    keep = edge_tokens if edge_tokens.size else np.zeros(1, np.int32)
    _check(_lib.peek_tree_canonical_ids(len(parent), parent.ctypes.data_as(_i32p), edge_offsets.ctypes.data_as(_i64p),
                                        keep.ctypes.data_as(_i32p), out.ctypes.data_as(_i32p)))
    return out


def peek_tree_from_sequences(tokens, offsets):
    """Raw cached sequences -> canonical tree description (parent, edge_offsets, edge_tokens)."""
    tokens, offsets = _np32(tokens), _np64(offsets)
    keep = tokens if tokens.size else np.zeros(1, np.int32)
    nn = ctypes.c_int32()
    P, O, T = _i32p(), _i64p(), _i32p()
    _check(_lib.peek_tree_from_sequences(keep.ctypes.data_as(_i32p), offsets.ctypes.data_as(_i64p),
                                         len(offsets) - 1, ctypes.byref(nn), ctypes.byref(P), ctypes.byref(O),
                                         ctypes.byref(T)))
    try:
        n = nn.value
        parent = np.ctypeslib.as_array(P, shape=(n,)).copy()
        eoff = np.ctypeslib.as_array(O, shape=(n + 1,)).copy()
        etok = np.ctypeslib.as_array(T, shape=(max(1, int(eoff[-1])),)).copy()[:int(eoff[-1])]
    finally:
        for p in (P, O, T):
            _lib.peek_free_host(ctypes.cast(p, _vp))
    return parent, eoff, etok


class Cache:
    """Owns a peek_cache handle (device CSR of a cache tree)."""

    def __init__(self, handle: int):
        self.handle = ctypes.c_void_p(handle)

    def free(self):
        if self.handle:
            _check(_lib.peek_cache_free(self.handle))
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            if self.handle:
                _lib.peek_cache_free(self.handle)
        except Exception:
            pass

    def stats(self) -> dict:
        return peek_cache_stats(self)


def peek_cache_build(parent, edge_offsets, edge_tokens, stream=None):
    """Host tree description -> (Cache, canon_id[int32, num_nodes])."""
    parent, edge_offsets, edge_tokens = _np32(parent), _np64(edge_offsets), _np32(edge_tokens)
    keep = edge_tokens if edge_tokens.size else np.zeros(1, np.int32)
    canon = np.empty(len(parent), dtype=np.int32)
    out = ctypes.c_void_p()
    _check(_lib.peek_cache_build(len(parent), parent.ctypes.data_as(_i32p), edge_offsets.ctypes.data_as(_i64p),
                                 keep.ctypes.data_as(_i32p), _stream(stream), ctypes.byref(out),
                                 canon.ctypes.data_as(_i32p)))
    return Cache(out.value), canon


def peek_cache_stats(cache: Cache) -> dict:
    nn, et, md, db = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    mf = ctypes.c_int32()
    _check(_lib.peek_cache_stats(cache.handle, ctypes.byref(nn), ctypes.byref(et), ctypes.byref(mf),
                                 ctypes.byref(md), ctypes.byref(db)))
    return {"num_nodes": nn.value, "num_edge_tokens": et.value, "max_fanout": mf.value,
            "max_depth": md.value, "device_bytes": db.value}


def peek_cache_export(cache: Cache) -> dict:
    n = peek_cache_stats(cache)["num_nodes"]
    out = {k: np.empty(n, dtype=np.int32) for k in ("parent", "depth", "edge_len", "subtree_end")}
    _check(_lib.peek_cache_export(cache.handle, *(out[k].ctypes.data_as(_i32p)
                                                  for k in ("parent", "depth", "edge_len", "subtree_end"))))
    return out


def peek_cache_free(cache: Cache):
    cache.free()


def peek_lpm_batch(cache: Cache, tokens, offsets, block_size: int, h, last_node=None, match_len=None,
                   stream=None):
    """tokens int32[*], offsets int64[n+1], outputs int32[n]: all torch tensors on the device."""
    import torch
    n = _queue_n(offsets)
    i32 = torch.int32
    _check(_lib.peek_lpm_batch(cache.handle, n, _arg(tokens, "tokens", i32), _arg(offsets, "offsets"),
                               int(block_size), _arg(h, "h", i32, n), _arg(last_node, "last_node", i32, n),
                               _arg(match_len, "match_len", i32, n), _stream(stream)))


def peek_queue_signals_workspace(n: int, num_nodes: int) -> int:
    return int(_lib.peek_queue_signals_workspace(int(n), int(num_nodes)))


def peek_queue_signals(cache, tokens, offsets, last_node, match_len, threshold: int, cluster_id, cluster_size,
                       demand, workspace, stream=None):
    """cluster_id/cluster_size int32[n], demand int32[num_nodes], workspace uint8 tensor; torch tensors.
    last_node/match_len: peek_lpm_batch outputs for the same prompts (or None)."""
    import torch
    n = _queue_n(offsets)
    i32 = torch.int32
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check(_lib.peek_queue_signals(None if cache is None else cache.handle, n, _arg(tokens, "tokens", i32),
                                   _arg(offsets, "offsets"), _arg(last_node, "last_node", i32, n),
                                   _arg(match_len, "match_len", i32, n), int(threshold),
                                   _arg(cluster_id, "cluster_id", i32, n), _arg(cluster_size, "cluster_size", i32, n),
                                   _arg(demand, "demand", i32, _num_nodes(cache)), _arg(workspace, "workspace"),
                                   ws_bytes, _stream(stream)))


PEEK_NOALLOC_SCRATCH_BYTES = 32 << 20


def peek_queue_signals_noalloc(cache, tokens, offsets, last_node, match_len, threshold: int, cluster_id,
                               cluster_size, demand, stream=None):
    """peek_queue_signals with the library's static scratch instead of a workspace (allocates nothing)."""
    import torch
    n = _queue_n(offsets)
    i32 = torch.int32
    _check(_lib.peek_queue_signals_noalloc(None if cache is None else cache.handle, n, _arg(tokens, "tokens", i32),
                                           _arg(offsets, "offsets"), _arg(last_node, "last_node", i32, n),
                                           _arg(match_len, "match_len", i32, n), int(threshold),
                                           _arg(cluster_id, "cluster_id", i32, n),
                                           _arg(cluster_size, "cluster_size", i32, n),
                                           _arg(demand, "demand", i32, _num_nodes(cache)), _stream(stream)))


def peek_clpm_signals(cache, tokens, offsets, h, last_node, match_len, threshold: int, tau: int, theta: int,
                      cluster_id, cluster_size, demand, score, section, has_sharing, workspace, stream=None):
    """peek_queue_signals plus the ancestor score (int64[n]), the section (int32[n]) and has_sharing (int32[1]);
    torch tensors, any of score/section/has_sharing may be None."""
    import torch
    n = _queue_n(offsets)
    i32 = torch.int32
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check(_lib.peek_clpm_signals(None if cache is None else cache.handle, n, _arg(tokens, "tokens", i32),
                                  _arg(offsets, "offsets"), _arg(h, "h", i32, n), _arg(last_node, "last_node", i32, n),
                                  _arg(match_len, "match_len", i32, n), int(threshold), int(tau), int(theta),
                                  _arg(cluster_id, "cluster_id", i32, n), _arg(cluster_size, "cluster_size", i32, n),
                                  _arg(demand, "demand", i32, _num_nodes(cache)), _arg(score, "score", torch.int64, n),
                                  _arg(section, "section", i32, n), _arg(has_sharing, "has_sharing", i32, 1),
                                  _arg(workspace, "workspace"), ws_bytes, _stream(stream)))


def peek_evict_rank_workspace(num_nodes: int) -> int:
    return int(_lib.peek_evict_rank_workspace(int(num_nodes)))


def peek_evict_rank(cache, demand, score, order, workspace, stream=None):
    """Eviction score int64[num_nodes] and victim order int32[num_nodes-1] from demand int32[num_nodes];
    torch tensors, score or order may be None."""
    import torch
    nn = _num_nodes(cache)
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check(_lib.peek_evict_rank(cache.handle, _arg(demand, "demand", torch.int32, nn),
                                _arg(score, "score", torch.int64, nn), _arg(order, "order", torch.int32, nn - 1),
                                _arg(workspace, "workspace"), ws_bytes, _stream(stream)))


class BlockTable:
    """Owns a peek_block_table handle (device table of chained block hashes)."""

    def __init__(self, handle: int):
        self.handle = ctypes.c_void_p(handle)

    def free(self):
        if self.handle:
            _check(_lib.peek_block_table_free(self.handle))
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            if self.handle:
                _lib.peek_block_table_free(self.handle)
        except Exception:
            pass

    def stats(self) -> dict:
        return peek_block_table_stats(self)


def peek_block_table_build(parent, edge_offsets, edge_tokens, block_size: int, stream=None) -> BlockTable:
    """Host tree description -> BlockTable on the current device."""
    parent, edge_offsets, edge_tokens = _np32(parent), _np64(edge_offsets), _np32(edge_tokens)
    keep = edge_tokens if edge_tokens.size else np.zeros(1, np.int32)
    out = ctypes.c_void_p()
    _check(_lib.peek_block_table_build(len(parent), parent.ctypes.data_as(_i32p), edge_offsets.ctypes.data_as(_i64p),
                                       keep.ctypes.data_as(_i32p), int(block_size), _stream(stream),
                                       ctypes.byref(out)))
    return BlockTable(out.value)


def peek_block_table_stats(table: BlockTable) -> dict:
    nb, ns = ctypes.c_int64(), ctypes.c_int64()
    bs = ctypes.c_int32()
    _check(_lib.peek_block_table_stats(table.handle, ctypes.byref(nb), ctypes.byref(ns), ctypes.byref(bs)))
    return {"num_blocks": nb.value, "num_slots": ns.value, "block_size": bs.value}


def peek_block_table_free(table: BlockTable):
    table.free()


def peek_block_lpm_batch(table, tokens, offsets, h, stream=None):
    """Hashed-block hit int32[n] of every prompt; tokens int32[*], offsets int64[n+1]: torch tensors on the device."""
    import torch
    n = _queue_n(offsets)
    _check(_lib.peek_block_lpm_batch(None if table is None else table.handle, n, _arg(tokens, "tokens", torch.int32),
                                     _arg(offsets, "offsets"), _arg(h, "h", torch.int32, n), _stream(stream)))


def peek_offline_order_workspace(n: int) -> int:
    return int(_lib.peek_offline_order_workspace(int(n)))


def peek_offline_order(tokens, offsets, depth_limit: int, perm, workspace, stream=None):
    """PEEK-offline Phase 1 permutation int32[n] of the prompts' first depth_limit tokens; torch tensors on the
    device."""
    import torch
    n = _queue_n(offsets)
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check(_lib.peek_offline_order(n, _arg(tokens, "tokens", torch.int32), _arg(offsets, "offsets"), int(depth_limit),
                                   _arg(perm, "perm", torch.int32, n), _arg(workspace, "workspace"), ws_bytes,
                                   _stream(stream)))


PEEK_TYPE_BF16 = 0
PEEK_TYPE_F16 = 1
PEEK_TYPE_F8E4M3 = 2
PEEK_TYPE_I8 = 3

_ROW_TYPES = {torch.bfloat16: PEEK_TYPE_BF16, torch.float16: PEEK_TYPE_F16}
_PAGE_TYPES = {torch.float8_e4m3fn: PEEK_TYPE_F8E4M3, torch.int8: PEEK_TYPE_I8}


class _PoolStruct(ctypes.Structure):
    _fields_ = [("d_pages", _vp), ("d_scales", _vp), ("num_pages", _i64), ("kv_heads", _i32), ("block_size", _i32),
                ("head_dim", _i32), ("type", _i32)]


class KVPool:
    """The cache's contents: pages [num_pages, 2, kv_heads, block_size, head_dim] of 8-bit codes (K at 0, V at 1;
    torch.float8_e4m3fn or torch.int8) and scales float32 [num_pages, 2, kv_heads], tensors of the caller's. They stay
    the pool's: other tensors make another pool."""

    def __init__(self, pages, scales):
        if pages.dtype not in _PAGE_TYPES:
            raise TypeError(f"pages must be torch.float8_e4m3fn or torch.int8, got {pages.dtype}")
        if pages.dim() != 5 or pages.shape[1] != 2:
            raise ValueError("pages must be [num_pages, 2, kv_heads, block_size, head_dim]")
        if scales.shape != pages.shape[:3]:
            raise ValueError(f"scales must be {tuple(pages.shape[:3])}, got {tuple(scales.shape)}")
        self._pages, self._scales = pages, scales
        self.num_pages, _, self.kv_heads, self.block_size, self.head_dim = pages.shape
        p, s = _arg(pages, "pages"), _arg(scales, "scales", torch.float32)
        self._struct = _PoolStruct(p, s, self.num_pages, self.kv_heads, self.block_size, self.head_dim,
                                   _PAGE_TYPES[pages.dtype])
        self._ref = ctypes.addressof(self._struct)

    @property
    def pages(self):
        return self._pages

    @property
    def scales(self):
        return self._scales

    @classmethod
    def empty(cls, num_pages: int, kv_heads: int, block_size: int, head_dim: int, dtype=torch.float8_e4m3fn,
              device="cuda") -> "KVPool":
        """A pool of new memory. Pages hold nothing until peek_kv_append writes them."""
        pages = torch.empty((num_pages, 2, kv_heads, block_size, head_dim), dtype=dtype, device=device)
        return cls(pages, torch.ones((num_pages, 2, kv_heads), dtype=torch.float32, device=device))


def _rows(t, name: str, dtype, heads: int | None = None, dim: int | None = None, tokens: int | None = None):
    """Pointer and strides of rows of heads [tokens, heads, dim], whose last dimension is contiguous."""
    shape = t.shape
    if len(shape) != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    n, h, d = shape
    if (heads is not None and h != heads) or (dim is not None and d != dim) or (tokens is not None and n != tokens):
        raise ValueError(f"{name} must be [{tokens}, {heads}, {dim}], got {list(t.shape)}")
    token, head, one = t.stride()
    if one != 1 and d > 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    # a dimension of one element has no stride that matters
    return t.data_ptr(), token if n > 1 else 0, head if h > 1 else 0


def _row_type(t, name: str) -> int:
    if t.dtype not in _ROW_TYPES:
        raise TypeError(f"{name} must be torch.bfloat16 or torch.float16, got {t.dtype}")
    return _ROW_TYPES[t.dtype]


def _table(t, n: int):
    """Pointer, width and row stride of a block table int32[n, max_blocks]; a view of its leading columns is one too."""
    if t.dtype != torch.int32:
        raise TypeError(f"block_table must be torch.int32, got {t.dtype}")
    if t.dim() != 2 or t.shape[0] != n:
        raise ValueError(f"block_table must be [{n}, max_blocks], got {list(t.shape)}")
    width = t.shape[1]
    if width > 1 and t.stride(1) != 1:
        raise ValueError("block_table's rows must be contiguous")
    if n > 1 and width > 0 and t.stride(0) < width:      # (one row expanded to all sequences, for one)
        raise ValueError("block_table's rows must not overlap")
    if not t.is_cuda:
        raise ValueError("block_table must be a device tensor")
    return t.data_ptr(), width, t.stride(0) if n > 1 and width > 0 else width


def _ws(workspace):
    return _arg(workspace, "workspace"), 0 if workspace is None else workspace.numel() * workspace.element_size()


def peek_kv_append(pool: KVPool, k, v, offsets, context, block_table, stream=None):
    """Quantises the K and V of new tokens into the pool. k, v [tokens, kv_heads, head_dim] (bfloat16 or float16, any
    token and head strides), offsets int64[n+1], context int32[n] (tokens cached before), block_table int32[n, *]."""
    n = _queue_n(offsets)
    kind = _row_type(k, "k")
    table = _table(block_table, n)
    _check(_lib.peek_kv_append(pool._ref, n, k.shape[0], kind, *_rows(k, "k", k.dtype, pool.kv_heads, pool.head_dim),
                               *_rows(v, "v", k.dtype, pool.kv_heads, pool.head_dim, k.shape[0]),
                               _arg(offsets, "offsets"), _arg(context, "context", torch.int32, n), *table,
                               _stream(stream)))


def peek_prefill_attention_workspace(n: int, num_tokens: int, q_heads: int, kv_heads: int, head_dim: int,
                                     max_context: int) -> int:
    return int(_lib.peek_prefill_attention_workspace(int(n), int(num_tokens), int(q_heads), int(kv_heads),
                                                     int(head_dim), int(max_context)))


def peek_prefill_attention(q, k, v, offsets, out, workspace, pool: KVPool | None = None, prefix=None,
                           block_table=None, scale: float | None = None, lse=None, stream=None):
    """Causal attention of packed prompts, each after its cached prefix. q, out [tokens, q_heads, head_dim], k, v
    [tokens, kv_heads, head_dim] (any token and head strides), offsets int64[n+1], prefix int32[n] (peek_lpm_batch's
    h) with the pool and block table that hold it; lse float32[tokens, q_heads] or None. scale: 1 / sqrt(head_dim)."""
    n = _queue_n(offsets)
    kind = _row_type(q, "q")
    tokens, q_heads, dim = q.shape if q.dim() == 3 else (0, 0, 0)
    kv_heads = k.shape[1] if k.dim() == 3 else 0
    if (pool is None) != (prefix is None) or (pool is None) != (block_table is None):
        raise ValueError("pool, prefix and block_table must be given together")
    table = (None, 0, 0) if pool is None else _table(block_table, n)
    _check(_lib.peek_prefill_attention(
        None if pool is None else pool._ref, n, tokens, kind, q_heads, kv_heads, dim, *_rows(q, "q", q.dtype),
        *_rows(k, "k", q.dtype, None, dim, tokens), *_rows(v, "v", q.dtype, kv_heads, dim, tokens),
        _arg(offsets, "offsets"), _arg(prefix, "prefix", torch.int32, n), *table,
        dim ** -0.5 if scale is None else scale, *_rows(out, "out", q.dtype, q_heads, dim, tokens),
        _row_arg(lse, "lse", torch.float32, tokens, q_heads), *_ws(workspace), _stream(stream)))


def peek_decode_attention_workspace(pool: KVPool, n: int, q_heads: int, max_blocks: int, mass: bool = False) -> int:
    return int(_lib.peek_decode_attention_workspace(pool._ref, int(n), int(q_heads), int(max_blocks), int(mass)))


def peek_decode_attention(pool: KVPool, q, context, block_table, out, workspace, scale: float | None = None, lse=None,
                          mass_in=None, mass=None, stream=None):
    """Attention of one token per sequence over the context[r] first tokens of its pages. q, out [n, q_heads,
    head_dim], context int32[n], block_table int32[n, max_blocks]; lse float32[n, q_heads] or None; mass
    float32[n, kv_heads, max_blocks] or None receives mass_in (or 0) plus the weight on every block."""
    n = q.shape[0]
    kind = _row_type(q, "q")
    q_heads = q.shape[1] if q.dim() == 3 else 0
    table = _table(block_table, n)
    masses = pool.kv_heads, table[1]
    _check(_lib.peek_decode_attention(
        pool._ref, n, kind, q_heads, *_rows(q, "q", q.dtype, None, pool.head_dim),
        _arg(context, "context", torch.int32, n), *table, pool.head_dim ** -0.5 if scale is None else scale,
        *_rows(out, "out", q.dtype, q_heads, pool.head_dim, n), _row_arg(lse, "lse", torch.float32, n, q_heads),
        _row_arg(mass_in, "mass_in", torch.float32, n, *masses), _row_arg(mass, "mass", torch.float32, n, *masses),
        *_ws(workspace), _stream(stream)))


def peek_kv_evict_workspace(n: int, kv_heads: int, max_blocks: int) -> int:
    return int(_lib.peek_kv_evict_workspace(int(n), int(kv_heads), int(max_blocks)))


def peek_kv_evict(context, block_table, mass, keep, block_size: int, sink: int, recent: int, context_out,
                  block_table_out, mass_out, freed, num_freed, workspace, stream=None):
    """Drops the blocks of least mass from sequences with more than keep[r] of them. context, keep, context_out,
    num_freed int32[n]; block_table int32[n, max_blocks] (rows of any stride), block_table_out and freed the same,
    contiguous; mass, mass_out float32[n, kv_heads, max_blocks]."""
    i32 = torch.int32
    if mass.dim() != 3:
        raise ValueError("mass must be [n, kv_heads, max_blocks]")
    n, heads, width = mass.shape
    table = _table(block_table, n)
    if table[1] != width:
        raise ValueError(f"block_table has {table[1]} columns, mass {width}")
    _check(_lib.peek_kv_evict(n, heads, int(block_size), _arg(context, "context", i32, n), *table,
                              _arg(mass, "mass", torch.float32), _arg(keep, "keep", i32, n), int(sink), int(recent),
                              _arg(context_out, "context_out", i32, n),
                              _row_arg(block_table_out, "block_table_out", i32, n, width),
                              _row_arg(mass_out, "mass_out", torch.float32, n, heads, width),
                              _row_arg(freed, "freed", i32, n, width), _arg(num_freed, "num_freed", i32, n),
                              *_ws(workspace), _stream(stream)))


PEEK_ROTARY_PLAIN = 0
PEEK_ROTARY_LINEAR = 1
PEEK_ROTARY_BASE = 2
PEEK_ROTARY_TURNS = 3
PEEK_ROTARY_RAMP = 4


class _RotaryStruct(ctypes.Structure):
    _fields_ = [("d_freq", _vp), ("rot_dim", _i32), ("interleaved", _i32), ("magnitude", ctypes.c_float),
                ("eps", ctypes.c_float), ("d_q_norm", _vp), ("d_k_norm", _vp)]


# The current device's number without the check that torch is initialised, where this torch has that.
_raw_device = getattr(torch._C, "_cuda_getDevice", None)
_devices = None     # how many there are, once asked


def _place(stream, *tensors):
    """The stream's handle, after refusing tensors of a device other than the current one, where the kernels run."""
    global _devices
    fast = _raw_device is not None and _raw_stream is not None and torch.cuda.is_initialized()
    now = _raw_device() if fast else torch.cuda.current_device()
    if _devices is None:
        _devices = torch.cuda.device_count()
    if _devices > 1:            # (of a single device, as every tensor's own check has found, they all are)
        for t in tensors:
            if t is not None and t.get_device() != now:
                raise ValueError(f"tensors must be on the current device (cuda:{now}), got one on {t.device}")
    if stream is None:
        return _raw_stream(now) if fast else torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _exact_arg(t, name: str, dtype, *shape: int):
    """As _arg, of this shape and no other."""
    if t is None:
        return None
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return _arg(t, name, dtype)


def peek_rotary_frequencies(rot_dim: int, base: float = 10000.0, scaling: int = PEEK_ROTARY_PLAIN, factor: float = 1.0,
                            trained: float = 0.0, low: float = 1.0, high: float = 4.0) -> np.ndarray:
    """Radians a token of every pair, float64[rot_dim / 2], on the host: base ** (-2 i / rot_dim), scaled for contexts
    `factor` times as long as trained (PEEK_ROTARY_LINEAR, _BASE, _TURNS, _RAMP)."""
    out = np.empty(max(0, int(rot_dim)) // 2, dtype=np.float64)
    _check(_lib.peek_rotary_frequencies(int(rot_dim), base, int(scaling), factor, trained, low, high,
                                        out.ctypes.data_as(ctypes.POINTER(ctypes.c_double))))
    return out


def peek_rotate_append(q, k, v, offsets, context, freq, q_out, k_out=None, pool: KVPool | None = None,
                       block_table=None, interleaved: bool = False, magnitude: float = 1.0, q_norm=None, k_norm=None,
                       eps: float = 1e-6, stream=None):
    """Norms and rotates every head of q and k by its token's position, and appends K and V to the pool. q, q_out
    [tokens, q_heads, head_dim] (both None: only K and V), k, v, k_out [tokens, kv_heads, head_dim] (any token and head
    strides; an output may be its own input), offsets int64[n+1], context int32[n] (tokens before), freq float64
    [rot_dim / 2] or None, q_norm, k_norm [head_dim] of the rows' type or None. Without a pool (v and block_table None)
    only q_out and k_out are written; without k (None, as k_out) only q_out."""
    n = _queue_n(offsets)
    if k is None and q is None:
        raise ValueError("k and q are both None")
    if k is None and (pool is not None or k_out is not None):
        raise ValueError("k must be given with a pool or k_out")
    of, name = (q, "q") if k is None else (k, "k")
    kind, dtype = _row_type(of, name), of.dtype
    if of.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    tokens, kv_heads, dim = of.shape
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out must be given together")
    if (pool is None) != (v is None) or (pool is None) != (block_table is None):
        raise ValueError("pool, v and block_table must be given together")
    if pool is None and k_out is None and k is not None:
        raise ValueError("k needs a pool or k_out")
    q_heads = 0 if q is None else q.shape[1] if q.dim() == 3 else -1
    rows_q = rows_q_out = rows_k = rows_v = rows_k_out = table = (None, 0, 0)
    if k is None:
        kv_heads = 1                    # (of no rows)
    else:
        rows_k = _rows(k, "k", dtype)
    if q is not None:
        rows_q = _rows(q, "q", dtype, None, dim, tokens)
        rows_q_out = _rows(q_out, "q_out", dtype, q_heads, dim, tokens)
    if v is not None:
        rows_v = _rows(v, "v", dtype, kv_heads, dim, tokens)
        table = _table(block_table, n)
    if k_out is not None:
        rows_k_out = _rows(k_out, "k_out", dtype, kv_heads, dim, tokens)
    if (q is not None and rows_q_out[0] == rows_q[0] and rows_q_out != rows_q) or \
            (k_out is not None and rows_k_out[0] == rows_k[0] and rows_k_out != rows_k):
        raise ValueError("an output in place of its input must have its strides")
    rot = 0 if freq is None else 2 * freq.numel()
    rotary = _RotaryStruct(_arg(freq, "freq", torch.float64), rot, int(bool(interleaved)), magnitude, eps,
                           _exact_arg(q_norm, "q_norm", dtype, dim), _exact_arg(k_norm, "k_norm", dtype, dim))
    at, ctx = _arg(offsets, "offsets"), _arg(context, "context", torch.int32, n)
    on = _place(stream, q, k, v, offsets, context, freq, q_out, k_out, block_table, q_norm, k_norm,
                None if pool is None else pool._pages)
    _check(_lib.peek_rotate_append(None if pool is None else pool._ref, n, tokens, kind, q_heads, kv_heads, dim,
                                   ctypes.addressof(rotary), *rows_q, *rows_k, *rows_v, at, ctx, *table, *rows_q_out,
                                   *rows_k_out, on))


def peek_kv_read(pool: KVPool, offsets, first, block_table, k_out, v_out, stream=None):
    """Tokens of the cache as rows: k_out, v_out [tokens, kv_heads, head_dim] (bfloat16 or float16, any token and head
    strides) receive, in rows offsets[r] .. offsets[r+1] (int64[n+1]), sequence r's tokens from first[r] on (int32[n])."""
    n = _queue_n(offsets)
    kind = _row_type(k_out, "k_out")
    table = _table(block_table, n)
    rows_k = _rows(k_out, "k_out", k_out.dtype, pool.kv_heads, pool.head_dim)
    rows_v = _rows(v_out, "v_out", k_out.dtype, pool.kv_heads, pool.head_dim, k_out.shape[0])
    at, begin = _arg(offsets, "offsets"), _arg(first, "first", torch.int32, n)
    on = _place(stream, pool._pages, offsets, first, block_table, k_out, v_out)
    _check(_lib.peek_kv_read(pool._ref, n, k_out.shape[0], kind, at, begin, *table, *rows_k, *rows_v, on))


def peek_shared_decode_attention_workspace(pool: KVPool, n: int, q_heads: int, max_blocks: int, groups: int) -> int:
    return int(_lib.peek_shared_decode_attention_workspace(pool._ref, int(n), int(q_heads), int(max_blocks),
                                                           int(groups)))


def peek_shared_decode_attention(pool: KVPool, q, context, block_table, group_offsets, shared, out, workspace,
                                 members=None, scale: float | None = None, lse=None, stream=None):
    """peek_decode_attention where groups of sequences have their first tokens in common, which are read once a group.
    Group g: the sequences members[group_offsets[g]] up to members[group_offsets[g + 1]] (members int32[n], None: in
    order; group_offsets int32[groups + 1]), which share their first shared[g] tokens (int32[groups]), read from the
    pages of the group's first."""
    n = q.shape[0]
    kind = _row_type(q, "q")
    q_heads = q.shape[1] if q.dim() == 3 else 0
    if group_offsets.dim() != 1 or group_offsets.numel() < 1:
        raise ValueError("group_offsets must be 1-D, of groups + 1 entries")
    groups, i32 = group_offsets.shape[0] - 1, torch.int32
    table = _table(block_table, n)
    on = _place(stream, pool._pages, q, context, block_table, group_offsets, shared, out, workspace, members, lse)
    _check(_lib.peek_shared_decode_attention(
        pool._ref, n, kind, q_heads, *_rows(q, "q", q.dtype, None, pool.head_dim), _arg(context, "context", i32, n),
        *table, groups, _arg(members, "members", i32, n), _arg(group_offsets, "group_offsets", i32),
        _arg(shared, "shared", i32, groups), pool.head_dim ** -0.5 if scale is None else scale,
        *_rows(out, "out", q.dtype, q_heads, pool.head_dim, n), _row_arg(lse, "lse", torch.float32, n, q_heads),
        *_ws(workspace), on))


def peek_kv_bounds(pool: KVPool, first, context, block_table, bounds, stream=None):
    """The largest and smallest key code of sequence r's blocks, from that of token first[r] on (None: from the first on)
    up to context[r] tokens, into bounds int8[num_pages, kv_heads, 2, head_dim]."""
    n = context.shape[0]
    table = _table(block_table, n)
    at = _exact_arg(bounds, "bounds", torch.int8, pool.num_pages, pool.kv_heads, 2, pool.head_dim)
    begin, ctx = _arg(first, "first", torch.int32, n), _arg(context, "context", torch.int32, n)
    on = _place(stream, pool._pages, first, context, block_table, bounds)
    _check(_lib.peek_kv_bounds(pool._ref, n, begin, ctx, *table, at, on))


def peek_block_select_workspace(pool: KVPool, n: int, max_blocks: int) -> int:
    return int(_lib.peek_block_select_workspace(pool._ref, int(n), int(max_blocks)))


def peek_block_select(pool: KVPool, bounds, q, context, block_table, sink: int, recent: int, context_out,
                      block_table_out, workspace, stream=None):
    """The blocks whose bounds promise the largest logits to each sequence's queries, for every kv head: block_table_out
    int32[n, kv_heads, keep] receives keep entries of block_table in order (the first `sink`, the last `recent`, and
    the best of the others), context_out int32[n, kv_heads] the tokens in them. q [n, q_heads, head_dim]."""
    n = q.shape[0]
    kind = _row_type(q, "q")
    q_heads = q.shape[1] if q.dim() == 3 else 0
    table = _table(block_table, n)
    if block_table_out.dim() != 3:
        raise ValueError("block_table_out must be [n, kv_heads, keep]")
    keep, i32 = block_table_out.shape[2], torch.int32
    at = _exact_arg(bounds, "bounds", torch.int8, pool.num_pages, pool.kv_heads, 2, pool.head_dim)
    on = _place(stream, pool._pages, bounds, q, context, block_table, context_out, block_table_out, workspace)
    _check(_lib.peek_block_select(
        pool._ref, at, n, kind, q_heads, *_rows(q, "q", q.dtype, None, pool.head_dim), _arg(context, "context", i32, n),
        *table, keep, int(sink), int(recent), _exact_arg(context_out, "context_out", i32, n, pool.kv_heads),
        _exact_arg(block_table_out, "block_table_out", i32, n, pool.kv_heads, keep), *_ws(workspace), on))


def peek_sparse_decode_attention_workspace(pool: KVPool, n: int, q_heads: int, keep: int) -> int:
    return int(_lib.peek_sparse_decode_attention_workspace(pool._ref, int(n), int(q_heads), int(keep)))


def peek_sparse_decode_attention(pool: KVPool, q, context, block_table, out, workspace, scale: float | None = None,
                                 lse=None, stream=None):
    """peek_decode_attention with a table and a length for every kv head, as peek_block_select leaves them: block_table
    int32[n, kv_heads, keep], context int32[n, kv_heads]."""
    n = q.shape[0]
    kind = _row_type(q, "q")
    q_heads = q.shape[1] if q.dim() == 3 else 0
    if block_table.dim() != 3:
        raise ValueError("block_table must be [n, kv_heads, keep]")
    keep, i32 = block_table.shape[2], torch.int32
    on = _place(stream, pool._pages, q, context, block_table, out, workspace, lse)
    _check(_lib.peek_sparse_decode_attention(
        pool._ref, n, kind, q_heads, *_rows(q, "q", q.dtype, None, pool.head_dim),
        _exact_arg(context, "context", i32, n, pool.kv_heads),
        _exact_arg(block_table, "block_table", i32, n, pool.kv_heads, keep), keep,
        pool.head_dim ** -0.5 if scale is None else scale, *_rows(out, "out", q.dtype, q_heads, pool.head_dim, n),
        _row_arg(lse, "lse", torch.float32, n, q_heads), *_ws(workspace), on))
