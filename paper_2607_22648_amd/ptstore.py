"""Python binding of the C ABI in include/ptstore.h (argument marshalling only).

The functions carry the C names and forward device pointers of torch tensors
plus the current HIP stream; every step of the work runs in the HIP library
``libptstore.so``. If the library has not been built this module raises at
import time: there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
import threading
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libptstore.so")

PTSTORE_OK, PTSTORE_ERR_INVALID, PTSTORE_ERR_FULL, PTSTORE_ERR_HIP, PTSTORE_ERR_NOMEM = 0, 1, 2, 3, 4
PTSTORE_FLAG_WEAK_HASH, PTSTORE_FLAG_COUNTERS, PTSTORE_FLAG_TIMING = 1, 2, 4
PTSTORE_FLAG_EVICT = 8
PTSTORE_FLAG_WEAK_TAGS = 16
PTSTORE_NOALLOC_MAX_ENTRIES = 1 << 20
KIND_GATHER, KIND_LOOKUP, KIND_SCATTER, KIND_INSERT, KIND_SELECT, KIND_EVICT = 0, 1, 2, 3, 4, 5
KIND_REPLICATE = 6
PTSTORE_KV_BF16, PTSTORE_KV_FP16, PTSTORE_KV_MXFP4 = 0, 1, 2


class ptstore_config_t(C.Structure):
    _fields_ = [("num_layers", C.c_int32), ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("block_tokens", C.c_int32), ("elem_bytes", C.c_int32),
                ("pool_blocks", C.c_int64), ("index_slots", C.c_int64),
                ("hash_seed", C.c_uint64), ("flags", C.c_uint32),
                ("host_blocks", C.c_int64), ("replica_blocks", C.c_int64),
                ("layer_chunk_bytes", C.c_void_p)]


class ptstore_stats_t(C.Structure):
    _fields_ = [(n, C.c_int64) for n in (
        "blocks_stored", "capacity", "index_slots", "block_bytes", "chunk_bytes", "full_events",
        "bad_entries", "probes", "token_compares", "cas_attempts", "cas_failures",
        "insert_fallbacks", "evictions", "clock", "index_rebuilds", "device_blocks", "replicas",
        "replica_copies")]


class ptstore_buffers_t(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("parent", C.c_void_p), ("tokens", C.c_void_p),
                ("slots", C.c_void_p), ("capacity", C.c_int64), ("index_slots", C.c_int64),
                ("freq", C.c_void_p), ("prio", C.c_void_p), ("host_pool", C.c_void_p),
                ("host_blocks", C.c_int64), ("device_blocks", C.c_int64), ("replica_of", C.c_void_p)]


class ptstore_kv_t(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("cache_blocks", C.c_int64),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("block_tokens", C.c_int32),
                ("kind", C.c_int32)]


class ptstore_attention_t(C.Structure):
    _fields_ = [("kv", ptstore_kv_t), ("q", C.c_void_p), ("q_token_stride", C.c_int64),
                ("q_head_stride", C.c_int64), ("out", C.c_void_p), ("out_token_stride", C.c_int64),
                ("out_head_stride", C.c_int64), ("lse", C.c_void_p), ("offsets", C.c_void_p),
                ("context", C.c_void_p), ("block_table", C.c_void_p), ("n_tokens", C.c_int64),
                ("R", C.c_int32), ("max_blocks", C.c_int32), ("q_heads", C.c_int32),
                ("scale", C.c_float), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class PTStoreError(RuntimeError):
    def __init__(self, fn: str, code: int, detail: str):
        super().__init__(f"{fn} failed: code {code} ({detail})")
        self.code = code


EXPORTS = ("ptstore_create", "ptstore_destroy", "ptstore_lookup", "ptstore_gather",
           "ptstore_lookup_gather", "ptstore_insert", "ptstore_scatter", "ptstore_stats",
           "ptstore_reset_counters", "ptstore_get_buffers", "ptstore_kernel_times",
           "ptstore_set_copy_shape", "ptstore_strerror", "ptstore_last_error",
           "ptstore_bandwidth_probe", "ptstore_replicate", "ptstore_gather_layers",
           "ptstore_scatter_layers", "ptstore_gather_prepare", "ptstore_gather_prepared",
           "ptstore_set_counters", "ptstore_set_timing", "ptstore_lookup_gather_noalloc",
           "ptstore_set_timing_kinds",
           "ptstore_insert_sync", "ptstore_kv_slab_bytes", "ptstore_block_tables",
           "ptstore_kv_append", "ptstore_kv_read", "ptstore_attention_workspace",
           "ptstore_attention")


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m "
                          "paper_2607_22648_amd.build or __graft_entry__.build())")
    lib = C.CDLL(LIB_PATH)
    p, i32, i64, d = C.c_void_p, C.c_int32, C.c_int64, C.c_double
    sig = {
        "ptstore_create": [C.POINTER(ptstore_config_t), C.POINTER(C.c_void_p)],
        "ptstore_destroy": [p],
        "ptstore_lookup": [p, p, p, i64, i32, i32, p, p, p],
        "ptstore_gather": [p, p, p, p, i32, i32, p, i64, p],
        "ptstore_lookup_gather": [p, p, p, i64, i32, i32, p, p, p, p, i64, p],
        "ptstore_lookup_gather_noalloc": [p, p, p, i64, i32, i32, p, p, p, p, i64, p],
        "ptstore_insert": [p, p, p, i64, i32, i32, p, p, p, p],
        "ptstore_insert_sync": [p, p, p, i64, i32, i32, p, p, p, p],
        "ptstore_scatter": [p, p, p, p, i32, i32, p, i64, p],
        "ptstore_stats": [p, C.POINTER(ptstore_stats_t)],
        "ptstore_reset_counters": [p],
        "ptstore_set_counters": [p, C.c_int],
        "ptstore_set_timing": [p, C.c_int],
        "ptstore_set_timing_kinds": [p, C.c_uint32],
        "ptstore_get_buffers": [p, C.POINTER(ptstore_buffers_t)],
        "ptstore_kernel_times": [p, i32, C.POINTER(d), C.POINTER(i64)],
        "ptstore_set_copy_shape": [p, i32, i32, i32],
        "ptstore_bandwidth_probe": [i32, p, p, i64, p],
        "ptstore_replicate": [p, p],
        "ptstore_gather_layers": [p, p, p, p, i32, i32, i32, i32, p, i64, p],
        "ptstore_scatter_layers": [p, p, p, p, i32, i32, i32, i32, p, i64, p],
        "ptstore_gather_prepare": [p, p, p, p, i32, i32, i64, p],
        "ptstore_gather_prepared": [p, i32, i32, p, i64, p],
        "ptstore_kv_slab_bytes": [i32, i32, i32, i32, C.POINTER(i64)],
        "ptstore_block_tables": [p, i64, p, p, i32, i32, i32, p, i64, p, p, p, p, p, p, p],
        "ptstore_kv_append": [C.POINTER(ptstore_kv_t), p, i64, i64, p, i64, i64, p, i64, p],
        "ptstore_kv_read": [C.POINTER(ptstore_kv_t), p, i64, i64, p, i64, i64, p, i64, p],
        "ptstore_attention_workspace": [C.POINTER(ptstore_kv_t), C.POINTER(i64)],
        "ptstore_attention": [C.POINTER(ptstore_attention_t), p],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = C.c_int
    lib.ptstore_strerror.argtypes = [C.c_int]
    lib.ptstore_strerror.restype = C.c_char_p
    lib.ptstore_last_error.argtypes = []
    lib.ptstore_last_error.restype = C.c_char_p
    return lib


_lib = _load()


def lib() -> C.CDLL:
    return _lib


def _check(fn: str, rc: int):
    if rc != PTSTORE_OK:
        raise PTStoreError(fn, rc, _lib.ptstore_last_error().decode())


def _dev(t: Optional[torch.Tensor], dtype, name: str) -> int:
    if t is None:
        return 0
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _arg(t: torch.Tensor, dtype, n: int, name: str) -> int:
    """The address of a required array of at least n elements: _dev and _need in one, since a short
    call's checks are a part of its time."""
    if t is not None and t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.numel() >= n:
        return t.data_ptr()
    _need(t, n, name)
    return _dev(t, dtype, name)


def _need(t: Optional[torch.Tensor], n: int, name: str) -> None:
    """The device arrays a call reads or writes are sized by R and max_blocks;
    the library cannot see an allocation's size, so it is checked here."""
    if t is None:
        if n:
            raise ValueError(f"{name} is required")
        return
    if t.numel() < n:
        raise ValueError(f"{name} holds {t.numel()} elements, the call needs {n}")


def _rows(ids: torch.Tensor, name: str = "ids") -> Tuple[int, int]:
    if ids.dim() != 2:
        raise ValueError(f"{name} must be [R, max_blocks], got shape {tuple(ids.shape)}")
    R, max_blocks = ids.shape
    return R, max_blocks


def _requests(offsets: torch.Tensor) -> int:
    if offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("offsets must be a 1-D tensor of R + 1 entries")
    return offsets.numel() - 1


def _table(offsets: torch.Tensor, block_table: torch.Tensor) -> Tuple[int, int]:
    R, maxb = _rows(block_table, "block_table")
    if offsets.numel() != R + 1 or offsets.dim() != 1:
        raise ValueError(f"block_table has {R} rows, the batch {_requests(offsets)} requests")
    return R, maxb


# The current stream's handle alone: building a torch.cuda.Stream to read it
# from takes longer than the rest of a short call's checks (a load of one small
# request 16.6 us with it, 13.9 without). The function is not public: where a
# torch release lacks it, the stream object is built.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


# ---------------------------------------------------------------------------
# C entry points under their own names
# ---------------------------------------------------------------------------

def ptstore_create(cfg: ptstore_config_t) -> C.c_void_p:
    h = C.c_void_p()
    _check("ptstore_create", _lib.ptstore_create(C.byref(cfg), C.byref(h)))
    return h


def ptstore_destroy(h) -> None:
    _check("ptstore_destroy", _lib.ptstore_destroy(h))


def ptstore_lookup(h, tokens, offsets, max_blocks, m, ids, stream=None) -> None:
    R = _requests(offsets)
    _need(m, R, "m")
    _need(ids, R * max_blocks, "ids")
    _check("ptstore_lookup", _lib.ptstore_lookup(
        h, _dev(tokens, torch.int32, "tokens"), _dev(offsets, torch.int64, "offsets"),
        tokens.numel(), R, max_blocks, _dev(m, torch.int32, "m"), _dev(ids, torch.int32, "ids"),
        _stream(stream)))


def _cache_blocks(cache: torch.Tensor, block_bytes: int) -> int:
    """Cache blocks a flat paged cache holds (every layer's slabs of one block)."""
    nbytes = cache.numel() * cache.element_size()
    per = block_bytes
    if nbytes % per:
        raise ValueError("cache size is not a whole number of blocks")
    return nbytes // per


def ptstore_gather(h, ids, m, block_table, cache, cache_blocks, stream=None) -> None:
    R, maxb = _rows(ids)
    _need(m, R, "m")
    _need(block_table, R * maxb, "block_table")
    _check("ptstore_gather", _lib.ptstore_gather(
        h, _dev(ids, torch.int32, "ids"), _dev(m, torch.int32, "m"),
        _dev(block_table, torch.int32, "block_table"), R, maxb, _dev(cache, None, "cache"),
        cache_blocks, _stream(stream)))


def ptstore_gather_layers(h, ids, m, block_table, layer_begin, layer_end, cache, cache_blocks,
                          stream=None) -> None:
    R, maxb = _rows(ids)
    _need(m, R, "m")
    _need(block_table, R * maxb, "block_table")
    _check("ptstore_gather_layers", _lib.ptstore_gather_layers(
        h, _dev(ids, torch.int32, "ids"), _dev(m, torch.int32, "m"),
        _dev(block_table, torch.int32, "block_table"), R, maxb, layer_begin, layer_end,
        _dev(cache, None, "cache"), cache_blocks, _stream(stream)))


def ptstore_gather_prepare(h, ids, m, block_table, cache_blocks, stream=None) -> None:
    R, maxb = _rows(ids)
    _need(m, R, "m")
    _need(block_table, R * maxb, "block_table")
    _check("ptstore_gather_prepare", _lib.ptstore_gather_prepare(
        h, _dev(ids, torch.int32, "ids"), _dev(m, torch.int32, "m"),
        _dev(block_table, torch.int32, "block_table"), R, maxb, cache_blocks, _stream(stream)))


def ptstore_gather_prepared(h, layer_begin, layer_end, cache, cache_blocks, stream=None) -> None:
    _check("ptstore_gather_prepared", _lib.ptstore_gather_prepared(
        h, layer_begin, layer_end, _dev(cache, None, "cache"), cache_blocks, _stream(stream)))


def ptstore_scatter_layers(h, ids, created, block_table, layer_begin, layer_end, cache,
                           cache_blocks, stream=None) -> None:
    R, maxb = _rows(ids)
    _need(created, R * maxb, "created")
    _need(block_table, R * maxb, "block_table")
    _check("ptstore_scatter_layers", _lib.ptstore_scatter_layers(
        h, _dev(ids, torch.int32, "ids"), _dev(created, torch.uint8, "created"),
        _dev(block_table, torch.int32, "block_table"), R, maxb, layer_begin, layer_end,
        _dev(cache, None, "cache"), cache_blocks, _stream(stream)))


def ptstore_lookup_gather(h, tokens, offsets, max_blocks, m, ids, block_table, cache, cache_blocks,
                          stream=None) -> None:
    R = _requests(offsets)
    _need(m, R, "m")
    _need(ids, R * max_blocks, "ids")
    _need(block_table, R * max_blocks, "block_table")
    _check("ptstore_lookup_gather", _lib.ptstore_lookup_gather(
        h, _dev(tokens, torch.int32, "tokens"), _dev(offsets, torch.int64, "offsets"),
        tokens.numel(), R, max_blocks, _dev(m, torch.int32, "m"), _dev(ids, torch.int32, "ids"),
        _dev(block_table, torch.int32, "block_table"), _dev(cache, None, "cache"), cache_blocks,
        _stream(stream)))


def ptstore_lookup_gather_noalloc(h, tokens, offsets, max_blocks, m, ids, block_table, cache,
                                  cache_blocks, stream=None) -> None:
    R = _requests(offsets)
    _need(m, R, "m")
    _need(ids, R * max_blocks, "ids")
    _need(block_table, R * max_blocks, "block_table")
    _check("ptstore_lookup_gather_noalloc", _lib.ptstore_lookup_gather_noalloc(
        h, _dev(tokens, torch.int32, "tokens"), _dev(offsets, torch.int64, "offsets"),
        tokens.numel(), R, max_blocks, _dev(m, torch.int32, "m"), _dev(ids, torch.int32, "ids"),
        _dev(block_table, torch.int32, "block_table"), _dev(cache, None, "cache"), cache_blocks,
        _stream(stream)))


def ptstore_insert(h, tokens, offsets, max_blocks, m_out, ids, created, stream=None) -> None:
    R = _requests(offsets)
    _need(m_out, R, "m_out")
    _need(ids, R * max_blocks, "ids")
    _need(created, R * max_blocks, "created")
    _check("ptstore_insert", _lib.ptstore_insert(
        h, _dev(tokens, torch.int32, "tokens"), _dev(offsets, torch.int64, "offsets"),
        tokens.numel(), R, max_blocks, _dev(m_out, torch.int32, "m_out"),
        _dev(ids, torch.int32, "ids"), _dev(created, torch.uint8, "created"), _stream(stream)))


def ptstore_insert_sync(h, tokens, offsets, max_blocks, m_out, ids, created, stream=None) -> int:
    """Returns PTSTORE_OK, or PTSTORE_ERR_FULL when the insert refused blocks
    (its outputs are written either way); raises on any other error."""
    R = _requests(offsets)
    _need(m_out, R, "m_out")
    _need(ids, R * max_blocks, "ids")
    _need(created, R * max_blocks, "created")
    rc = _lib.ptstore_insert_sync(
        h, _dev(tokens, torch.int32, "tokens"), _dev(offsets, torch.int64, "offsets"),
        tokens.numel(), R, max_blocks, _dev(m_out, torch.int32, "m_out"),
        _dev(ids, torch.int32, "ids"), _dev(created, torch.uint8, "created"), _stream(stream))
    if rc != PTSTORE_ERR_FULL:
        _check("ptstore_insert_sync", rc)
    return rc


def ptstore_scatter(h, ids, created, block_table, cache, cache_blocks, stream=None) -> None:
    R, maxb = _rows(ids)
    _need(created, R * maxb, "created")
    _need(block_table, R * maxb, "block_table")
    _check("ptstore_scatter", _lib.ptstore_scatter(
        h, _dev(ids, torch.int32, "ids"), _dev(created, torch.uint8, "created"),
        _dev(block_table, torch.int32, "block_table"), R, maxb, _dev(cache, None, "cache"),
        cache_blocks, _stream(stream)))


def ptstore_stats(h) -> dict:
    s = ptstore_stats_t()
    _check("ptstore_stats", _lib.ptstore_stats(h, C.byref(s)))
    return {n: getattr(s, n) for n, _ in s._fields_}


def ptstore_replicate(h, stream=None) -> None:
    _check("ptstore_replicate", _lib.ptstore_replicate(h, _stream(stream)))


def ptstore_reset_counters(h) -> None:
    _check("ptstore_reset_counters", _lib.ptstore_reset_counters(h))


def ptstore_set_counters(h, on: bool) -> None:
    _check("ptstore_set_counters", _lib.ptstore_set_counters(h, 1 if on else 0))


def ptstore_set_timing(h, on: bool) -> None:
    _check("ptstore_set_timing", _lib.ptstore_set_timing(h, 1 if on else 0))


def ptstore_set_timing_kinds(h, kinds: int) -> None:
    _check("ptstore_set_timing_kinds", _lib.ptstore_set_timing_kinds(h, kinds))


def ptstore_get_buffers(h) -> ptstore_buffers_t:
    b = ptstore_buffers_t()
    _check("ptstore_get_buffers", _lib.ptstore_get_buffers(h, C.byref(b)))
    return b


def ptstore_kernel_times(h, kind: int) -> Tuple[float, int]:
    ms, n = C.c_double(), C.c_int64()
    _check("ptstore_kernel_times", _lib.ptstore_kernel_times(h, kind, C.byref(ms), C.byref(n)))
    return ms.value, n.value


def ptstore_set_copy_shape(h, chunks_per_group: int = 0, threads: int = 0, grid: int = 0) -> None:
    _check("ptstore_set_copy_shape", _lib.ptstore_set_copy_shape(h, chunks_per_group, threads,
                                                                  grid))


def ptstore_bandwidth_probe(kind: int, a, b, nbytes: int, stream=None) -> None:
    """a, b: device tensors, or integer addresses the device can access (such as
    the pinned host tier)."""
    pa = a if isinstance(a, int) else _dev(a, None, "a")
    pb = b if isinstance(b, int) else _dev(b, None, "b")
    _check("ptstore_bandwidth_probe", _lib.ptstore_bandwidth_probe(kind, pa, pb, nbytes,
                                                                   _stream(stream)))


def ptstore_strerror(code: int) -> str:
    return _lib.ptstore_strerror(code).decode()


def ptstore_last_error() -> str:
    return _lib.ptstore_last_error().decode()


def ptstore_kv_slab_bytes(kind: int, kv_heads: int, head_dim: int, block_tokens: int) -> int:
    n = C.c_int64()
    _check("ptstore_kv_slab_bytes", _lib.ptstore_kv_slab_bytes(kind, kv_heads, head_dim, block_tokens,
                                                               C.byref(n)))
    return n.value


def _block_tables(R, maxb, offsets, context, held, block_tokens, free_blocks, first, block_table, n, outputs,
                  stream) -> None:
    """outputs: the addresses of slots, positions, held_out and next_free."""
    i32, i64 = torch.int32, torch.int64
    rc = _lib.ptstore_block_tables(
        _arg(offsets, i64, R + 1, "offsets"), n, _arg(context, i32, R, "context"),
        None if held is None else _arg(held, i32, R, "held"), R, maxb, block_tokens,
        _arg(free_blocks, i32, 0, "free_blocks"), free_blocks.numel(),
        None if first is None else _arg(first, i64, 1, "first"),
        _arg(block_table, i32, 0, "block_table"), *outputs, _stream(stream))
    if rc:
        _check("ptstore_block_tables", rc)


def ptstore_block_tables(offsets, context, held, block_tokens, free_blocks, first, block_table, slots,
                         positions, held_out, next_free, stream=None) -> None:
    """n_tokens is the length of `slots`; `held`, `first` and `positions` may be None."""
    R, maxb = _table(offsets, block_table)
    n, i32, i64 = slots.numel(), torch.int32, torch.int64
    outputs = (_arg(slots, i64, 0, "slots"), None if positions is None else _arg(positions, i32, n, "positions"),
               _arg(held_out, i32, R, "held_out"), _arg(next_free, i64, 1, "next_free"))
    _block_tables(R, maxb, offsets, context, held, block_tokens, free_blocks, first, block_table, n, outputs,
                  stream)


_KV_DTYPES = {PTSTORE_KV_BF16: torch.bfloat16, PTSTORE_KV_FP16: torch.float16,
              PTSTORE_KV_MXFP4: torch.bfloat16}


def _token_rows(t: torch.Tensor, kv: ptstore_kv_t, heads: Optional[int], name: str) -> Tuple[int, int, int]:
    """Address and strides of a [tokens, heads, head_dim] tensor whose rows are contiguous."""
    want = _KV_DTYPES[kv.kind]
    if not t.is_cuda or t.dtype is not want or t.dim() != 3:
        raise ValueError(f"{name} must be a [tokens, heads, head_dim] device tensor of {want}")
    n, h, dim = t.shape
    if dim != kv.head_dim or (heads is not None and h != heads):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, the cache {kv.kv_heads} heads of "
                         f"{kv.head_dim}")
    token, head, one = t.stride()
    if one != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    # a dimension of one row may have any stride: none of its others is reached
    return t.data_ptr(), token if n > 1 else 0, head if h > 1 else 0


def _rows_of(kv, k, v, slots):
    n = slots.numel()
    kr, vr = _token_rows(k, kv, kv.kv_heads, "k"), _token_rows(v, kv, kv.kv_heads, "v")
    if k.shape[0] != n or v.shape[0] != n:
        raise ValueError(f"k and v hold {k.shape[0]} and {v.shape[0]} tokens, slots {n}")
    return (*kr, *vr, _arg(slots, torch.int64, n, "slots"), n)


def ptstore_kv_append(kv: ptstore_kv_t, k, v, slots, stream=None) -> None:
    _check("ptstore_kv_append", _lib.ptstore_kv_append(C.byref(kv), *_rows_of(kv, k, v, slots),
                                                       _stream(stream)))


def ptstore_kv_read(kv: ptstore_kv_t, k, v, slots, stream=None) -> None:
    _check("ptstore_kv_read", _lib.ptstore_kv_read(C.byref(kv), *_rows_of(kv, k, v, slots),
                                                   _stream(stream)))


def ptstore_attention_workspace(kv: ptstore_kv_t) -> int:
    n = C.c_int64()
    _check("ptstore_attention_workspace", _lib.ptstore_attention_workspace(C.byref(kv), C.byref(n)))
    return n.value


def _attention(kv, q, out_rows, lse: Optional[int], offsets, context, block_table, scale, workspace,
               stream) -> None:
    """out_rows: address and strides of an output of q's shape; lse: an address, or None."""
    R, maxb = _table(offsets, block_table)
    n, heads, _ = q.shape
    a = ptstore_attention_t(kv, *_token_rows(q, kv, None, "q"), *out_rows, lse,
                            _arg(offsets, torch.int64, R + 1, "offsets"),
                            _arg(context, torch.int32, R, "context"),
                            _arg(block_table, torch.int32, 0, "block_table"), n, R, maxb, heads, scale,
                            _arg(workspace, torch.uint8, 0, "workspace"), workspace.numel())
    rc = _lib.ptstore_attention(C.byref(a), stream)
    if rc:
        _check("ptstore_attention", rc)


def ptstore_attention(kv: ptstore_kv_t, q, out, lse, offsets, context, block_table, scale: float,
                      workspace, stream=None) -> None:
    """`lse` may be None; `workspace`: a uint8 tensor of ptstore_attention_workspace(kv) bytes."""
    _token_rows(q, kv, None, "q")
    n, heads, _ = q.shape
    rows = _token_rows(out, kv, heads, "out")
    if out.shape[0] != n:
        raise ValueError(f"out holds {out.shape[0]} tokens, q {n}")
    _attention(kv, q, rows, None if lse is None else _arg(lse, torch.float32, n * heads, "lse"), offsets,
               context, block_table, scale, workspace, _stream(stream))


# ---------------------------------------------------------------------------
# Convenience wrappers
# ---------------------------------------------------------------------------

@dataclass
class StoreShape:
    layers: int
    kv_heads: int
    head_dim: int
    block_tokens: int = 16
    elem_bytes: int = 2
    layer_chunk_bytes: Optional[Tuple[int, ...]] = None  # per-layer slab sizes, or uniform

    @property
    def chunk_bytes(self) -> int:
        """Slab bytes of layer 0 (of every layer when they are uniform)."""
        if self.layer_chunk_bytes:
            return int(self.layer_chunk_bytes[0])
        return self.kv_heads * self.block_tokens * self.head_dim * self.elem_bytes

    @property
    def block_bytes(self) -> int:
        if self.layer_chunk_bytes:
            return 2 * int(sum(self.layer_chunk_bytes))
        return self.layers * 2 * self.chunk_bytes


class PrefixStore:
    """A store on the current device; methods take device tensors."""

    def __init__(self, shape: StoreShape, pool_blocks: int, index_slots: int = 0,
                 hash_seed: int = 0x5EED, flags: int = 0, host_blocks: int = 0,
                 replica_blocks: int = 0):
        self.shape = shape
        lcb = None
        if shape.layer_chunk_bytes:
            lcb = (C.c_int64 * shape.layers)(*[int(x) for x in shape.layer_chunk_bytes])
        cfg = ptstore_config_t(shape.layers, shape.kv_heads, shape.head_dim, shape.block_tokens,
                               shape.elem_bytes, pool_blocks, index_slots, hash_seed, flags,
                               host_blocks, replica_blocks,
                               C.cast(lcb, C.c_void_p) if lcb is not None else None)
        self.h = ptstore_create(cfg)  # the slab-size array is read here and not kept
        self._replicas = replica_blocks

    def close(self):
        if getattr(self, "h", None):
            ptstore_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self) -> "PrefixStore":
        return self

    def __exit__(self, *exc) -> None:
        self.close()

    def cache_blocks(self, cache: torch.Tensor) -> int:
        return _cache_blocks(cache, self.shape.block_bytes)

    def lookup(self, tokens, offsets, max_blocks, m=None, ids=None, stream=None):
        R = offsets.numel() - 1
        dev = offsets.device
        m = torch.empty(R, dtype=torch.int32, device=dev) if m is None else m
        ids = torch.empty((R, max_blocks), dtype=torch.int32, device=dev) if ids is None else ids
        ptstore_lookup(self.h, tokens, offsets, max_blocks, m, ids, stream)
        return m, ids

    def gather(self, ids, m, block_table, cache, stream=None, layers=None):
        """layers = (begin, end): only those layers' slabs (None: all)."""
        if layers is None:
            ptstore_gather(self.h, ids, m, block_table, cache, self.cache_blocks(cache), stream)
        else:
            ptstore_gather_layers(self.h, ids, m, block_table, layers[0], layers[1], cache,
                                  self.cache_blocks(cache), stream)

    def lookup_gather(self, tokens, offsets, max_blocks, block_table, cache, m=None, ids=None,
                      stream=None):
        R = offsets.numel() - 1
        dev = offsets.device
        m = torch.empty(R, dtype=torch.int32, device=dev) if m is None else m
        ids = torch.empty((R, max_blocks), dtype=torch.int32, device=dev) if ids is None else ids
        ptstore_lookup_gather(self.h, tokens, offsets, max_blocks, m, ids, block_table, cache,
                              self.cache_blocks(cache), stream)
        return m, ids

    def lookup_gather_noalloc(self, tokens, offsets, max_blocks, block_table, cache, m, ids,
                              stream=None):
        """ptstore_lookup_gather_noalloc: the caller brings every output buffer."""
        ptstore_lookup_gather_noalloc(self.h, tokens, offsets, max_blocks, m, ids, block_table,
                                      cache, self.cache_blocks(cache), stream)
        return m, ids

    def insert(self, tokens, offsets, max_blocks, stream=None):
        R = offsets.numel() - 1
        dev = offsets.device
        m = torch.empty(R, dtype=torch.int32, device=dev)
        ids = torch.empty((R, max_blocks), dtype=torch.int32, device=dev)
        created = torch.empty((R, max_blocks), dtype=torch.uint8, device=dev)
        ptstore_insert(self.h, tokens, offsets, max_blocks, m, ids, created, stream)
        return m, ids, created

    def insert_sync(self, tokens, offsets, max_blocks, stream=None):
        """(rc, m, ids, created): rc is PTSTORE_OK or PTSTORE_ERR_FULL."""
        R = offsets.numel() - 1
        dev = offsets.device
        m = torch.empty(R, dtype=torch.int32, device=dev)
        ids = torch.empty((R, max_blocks), dtype=torch.int32, device=dev)
        created = torch.empty((R, max_blocks), dtype=torch.uint8, device=dev)
        rc = ptstore_insert_sync(self.h, tokens, offsets, max_blocks, m, ids, created, stream)
        return rc, m, ids, created

    def gather_prepare(self, ids, m, block_table, cache, stream=None):
        """List once the blocks a gather of (ids, m, block_table) into `cache` moves."""
        ptstore_gather_prepare(self.h, ids, m, block_table, self.cache_blocks(cache), stream)

    def gather_prepared(self, cache, layers, stream=None):
        """Copy layers[0] .. layers[1]-1 of the prepared blocks into `cache`."""
        ptstore_gather_prepared(self.h, layers[0], layers[1], cache, self.cache_blocks(cache), stream)

    def scatter(self, ids, created, block_table, cache, stream=None, layers=None):
        """layers = (begin, end): only those layers' slabs (None: all)."""
        if layers is None:
            ptstore_scatter(self.h, ids, created, block_table, cache, self.cache_blocks(cache),
                            stream)
        else:
            ptstore_scatter_layers(self.h, ids, created, block_table, layers[0], layers[1], cache,
                                   self.cache_blocks(cache), stream)

    def replicate(self, stream=None):
        ptstore_replicate(self.h, stream)

    def stats(self) -> dict:
        return ptstore_stats(self.h)

    def reset_counters(self):
        ptstore_reset_counters(self.h)

    def set_counters(self, on: bool):
        ptstore_set_counters(self.h, on)

    def set_timing(self, on: bool):
        ptstore_set_timing(self.h, on)

    def set_timing_kinds(self, kinds: int):
        """Events around the kernels of the kinds whose bit is set only."""
        ptstore_set_timing_kinds(self.h, kinds)

    def kernel_times(self, kind: int) -> Tuple[float, int]:
        return ptstore_kernel_times(self.h, kind)

    def set_copy_shape(self, chunks_per_group: int = 0, threads: int = 0, grid: int = 0):
        ptstore_set_copy_shape(self.h, chunks_per_group, threads, grid)

    def buffers(self) -> ptstore_buffers_t:
        return ptstore_get_buffers(self.h)

    def pool_tensor(self) -> torch.Tensor:
        """The device pool as a uint8 [rows, block_bytes] device tensor (no copy): the
        home of ids below device_blocks, then the replica slots."""
        b = self.buffers()
        rows = b.device_blocks + self._replicas
        n = rows * self.shape.block_bytes
        return _wrap_device(b.pool, n, torch.uint8).view(rows, self.shape.block_bytes)

    def host_tensor(self) -> torch.Tensor:
        """The pinned host tier as a uint8 [host_blocks, block_bytes] CPU tensor (no
        copy); row j holds block id device_blocks + j."""
        b = self.buffers()
        if not b.host_pool:
            raise ValueError("store has no host tier")
        n = b.host_blocks * self.shape.block_bytes
        arr = (C.c_uint8 * n).from_address(b.host_pool)
        return torch.frombuffer(arr, dtype=torch.uint8).view(b.host_blocks, self.shape.block_bytes)

    def block_bytes_of(self, ids) -> torch.Tensor:
        """Home bytes of the given block ids, [len(ids), block_bytes] on the device
        (device tier rows and host tier rows alike; a test helper)."""
        b = self.buffers()
        ids = torch.as_tensor(ids, dtype=torch.int64)
        dev = self.pool_tensor()
        on_dev = ids < b.device_blocks
        if bool(on_dev.all()):
            return dev[ids.to(dev.device)]
        out = torch.empty((ids.numel(), self.shape.block_bytes), dtype=torch.uint8, device=dev.device)
        if bool(on_dev.any()):
            out[on_dev.to(dev.device)] = dev[ids[on_dev].to(dev.device)]
        if bool((~on_dev).any()):
            torch.cuda.synchronize()  # host-tier rows are written by device kernels
            host = self.host_tensor()
            out[(~on_dev).to(dev.device)] = host[ids[~on_dev] - b.device_blocks].to(dev.device)
        return out

    def replica_map(self) -> torch.Tensor:
        """[host_blocks] int32 device tensor: replica slot of each host-tier block, or -1."""
        b = self.buffers()
        if not b.replica_of:
            raise ValueError("store has no replica slots")
        return _wrap_device(b.replica_of, b.host_blocks, torch.int32)

    def meta_tensors(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """(parent [capacity] int32, tokens [capacity, block_tokens] int32), device, no copy."""
        b = self.buffers()
        par = _wrap_device(b.parent, b.capacity, torch.int32)
        tok = _wrap_device(b.tokens, b.capacity * self.shape.block_tokens, torch.int32)
        return par, tok.view(b.capacity, self.shape.block_tokens)

    def evict_tensors(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """(access counts F, priorities H), each [capacity] int64, device, no copy
        (the values are unsigned 64-bit; they stay far below 2^63)."""
        b = self.buffers()
        if not b.freq:
            raise ValueError("store created without PTSTORE_FLAG_EVICT")
        return (_wrap_device(b.freq, b.capacity, torch.int64),
                _wrap_device(b.prio, b.capacity, torch.int64))


_CURRENT = contextlib.nullcontext()  # tensors for the current stream
_KV_KINDS = {"bf16": PTSTORE_KV_BF16, "fp16": PTSTORE_KV_FP16, "mxfp4": PTSTORE_KV_MXFP4}


class PagedCache:
    """A paged cache [layer][K|V][cache block][slab] on the current device, and the
    operators on it. ``data`` is what the store's loads and ``scatter`` take; a store
    for its blocks is made with ``shape``. ``kv_heads`` is a number, or one per layer.

    Outputs and workspaces that a call makes are made for the stream it runs on. Several host
    threads may use one cache."""

    def __init__(self, layers: int, kv_heads: Union[int, Sequence[int]], head_dim: int, cache_blocks: int,
                 block_tokens: int = 16, kind: str = "bf16", data: Optional[torch.Tensor] = None,
                 device="cuda"):
        if kind not in _KV_KINDS:
            raise ValueError(f"kind must be one of {sorted(_KV_KINDS)}, got {kind!r}")
        heads = [kv_heads] * layers if isinstance(kv_heads, int) else [int(h) for h in kv_heads]
        if layers < 1 or len(heads) != layers or cache_blocks < 0:
            raise ValueError("a cache has layers, a number of KV heads for each, and 0 or more blocks")
        self.kind, self.cache_blocks, self.block_tokens = kind, cache_blocks, block_tokens
        slabs = [ptstore_kv_slab_bytes(_KV_KINDS[kind], h, head_dim, block_tokens) for h in heads]
        # slabs of values only, all alike: the uniform store shape; else sizes by layer
        uniform = kind != "mxfp4" and len(set(heads)) == 1
        self.shape = StoreShape(layers, heads[0], head_dim, block_tokens, 2,
                                None if uniform else tuple(slabs))
        nbytes = 2 * cache_blocks * sum(slabs)
        if data is None:
            data = torch.empty(nbytes, dtype=torch.uint8, device=device)
        if not data.is_cuda or not data.is_contiguous() or data.numel() * data.element_size() != nbytes:
            raise ValueError(f"data must be a contiguous device tensor of {nbytes} bytes")
        self.data = data
        self.dtype = _KV_DTYPES[_KV_KINDS[kind]]
        self._workspaces = {}
        self._turn = threading.Lock()
        self._scale = head_dim ** -0.5
        self._planes = []
        at = data.data_ptr()
        for h, slab in zip(heads, slabs):
            self._planes.append(ptstore_kv_t(at, at + cache_blocks * slab, cache_blocks, h, head_dim,
                                             block_tokens, _KV_KINDS[kind]))
            at += 2 * cache_blocks * slab

    def layer(self, layer: int) -> ptstore_kv_t:
        """The K and V planes of a layer, as the C calls take them."""
        return self._planes[layer]

    @staticmethod
    def _on(stream):
        """A context in which tensors are allocated for `stream` (a torch stream or a raw handle)."""
        if stream is None:
            return _CURRENT
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream))
        return torch.cuda.stream(stream)

    def _workspace(self, stream, handle: int) -> torch.Tensor:
        """The workspace of a stream: one serves every layer, and the calls on it in turn (_turn).
        A graph, which may be replayed on any stream, gets its own."""
        with self._on(stream):
            graph = torch.cuda.is_current_stream_capturing()
            ws = None if graph else self._workspaces.get(handle)
            if ws is None:
                need = max(ptstore_attention_workspace(kv) for kv in self._planes)
                ws = torch.empty(need, dtype=torch.uint8, device=self.data.device)
                if not graph:
                    self._workspaces[handle] = ws
        return ws

    def tables(self, offsets, context, block_table, free_blocks, n_tokens: int, held=None, first=None,
               stream=None):
        """Give the batch's requests their blocks: fills the new entries of `block_table` and
        returns (slots, positions, held after, next free entry)."""
        R, maxb = _table(offsets, block_table)
        with self._on(stream):
            slots, next_free = offsets.new_empty(n_tokens), offsets.new_empty(1)
            positions, held_out = context.new_empty(n_tokens), context.new_empty(R)
        # offsets and context are checked to be int64 and int32 arrays on the device: so are these
        _block_tables(R, maxb, offsets, context, held, self.block_tokens, free_blocks, first, block_table,
                      n_tokens, (slots.data_ptr(), positions.data_ptr(), held_out.data_ptr(),
                                 next_free.data_ptr()), stream)
        return slots, positions, held_out, next_free

    def append(self, layer: int, k, v, slots, stream=None) -> None:
        """Write k, v [tokens, kv_heads, head_dim] to `slots` of a layer."""
        ptstore_kv_append(self._planes[layer], k, v, slots, stream)

    def read(self, layer: int, slots, stream=None):
        """The K and V that `slots` of a layer hold, [tokens, kv_heads, head_dim] each."""
        kv = self._planes[layer]
        n, heads, dim = slots.numel(), kv.kv_heads, kv.head_dim
        with self._on(stream):
            k = slots.new_empty((n, heads, dim), dtype=self.dtype)
            v = slots.new_empty((n, heads, dim), dtype=self.dtype)
        row = heads * dim
        rc = _lib.ptstore_kv_read(C.byref(kv), k.data_ptr(), row, dim, v.data_ptr(), row, dim,
                                  _arg(slots, torch.int64, n, "slots"), n, _stream(stream))
        if rc:
            _check("ptstore_kv_read", rc)
        return k, v

    def attend(self, layer: int, q, offsets, context, block_table, scale: Optional[float] = None, out=None,
               lse: bool = False, workspace=None, stream=None):
        """Causal attention of q [tokens, q_heads, head_dim] over a layer: out, or (out, lse).
        scale: 1 / sqrt(head_dim) unless given. workspace: one of the caller's,
        instead of the one that the cache keeps for the stream."""
        kv = self._planes[layer]
        handle = _stream(stream)
        if q.dim() != 3:
            raise ValueError(f"q must be [tokens, heads, head_dim], got shape {tuple(q.shape)}")
        n, heads, dim = q.shape
        scale = self._scale if scale is None else scale
        with self._on(stream):
            sums = q.new_empty((n, heads), dtype=torch.float32) if lse else None
            made = q.new_empty((n, heads, dim)) if out is None else None
        # An attention is several kernels that hand parts on in the workspace, and the library's call
        # lets other host threads run: those of two threads on one stream must not mix.
        with self._turn if workspace is None else _CURRENT:
            if workspace is None:
                workspace = self._workspace(stream, handle)
            if made is None:
                ptstore_attention(kv, q, out, sums, offsets, context, block_table, scale, workspace, handle)
            else:  # contiguous, and of the right shape and place
                out = made
                _attention(kv, q, (out.data_ptr(), heads * dim, dim), sums.data_ptr() if lse else None,
                           offsets, context, block_table, scale, workspace, handle)
        return (out, sums) if lse else out


class _CudaArray:
    def __init__(self, ptr: int, n: int, typestr: str):
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": typestr, "data": (ptr, False),
                                         "version": 2, "strides": None}


def _wrap_device(ptr: int, n: int, dtype) -> torch.Tensor:
    typestr = {torch.uint8: "|u1", torch.int32: "<i4", torch.int64: "<i8"}[dtype]
    return torch.as_tensor(_CudaArray(ptr, n, typestr), device="cuda")
