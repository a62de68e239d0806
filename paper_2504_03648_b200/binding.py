"""Thin ctypes binding of libaibx: one Python function per C entry point, same names without
the ``aibx_`` prefix.  Argument marshalling only - every step of the path runs in the CUDA
kernels behind the C ABI (include/aibx.h).  There is no CPU fallback: if the library has not
been built, loading fails with an error.

Tensors are torch CUDA tensors used purely as device memory; the current torch stream is
passed to every call.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libaibx.so")

OK = 0
ERR_INVALID, ERR_RANGE, ERR_FULL, ERR_CUDA, ERR_UNSUPPORTED, ERR_NOMEM, ERR_TIMEOUT = (
    -1, -2, -3, -4, -5, -6, -7)
NO_BLOCK = 0xFFFFFFFF
NO_POD = -1
TYPE_BF16, TYPE_FP16, TYPE_FP32, TYPE_E4M3 = range(4)
ROPE_HALF, ROPE_INTERLEAVED = range(2)
_TYPE_OF = {torch.bfloat16: TYPE_BF16, torch.float16: TYPE_FP16, torch.float32: TYPE_FP32}


class AibxError(RuntimeError):
    def __init__(self, call: str, code: int):
        self.code = code
        super().__init__("%s failed: %d (%s)" % (call, code, strerror(code)))


class RouteParams(C.Structure):
    _fields_ = [("w_prefix", C.c_int32), ("w_load", C.c_int32), ("threshold_pct", C.c_int32)]


class KVLayout(C.Structure):
    _fields_ = [
        ("layout", C.c_int32),
        ("num_layers", C.c_int32),
        ("num_kv_heads", C.c_int32),
        ("block_tokens", C.c_int32),
        ("head_dim", C.c_int32),
        ("elem_bytes", C.c_int32),
        ("num_blocks", C.c_uint32),
    ]

    @property
    def tile_bytes(self) -> int:
        return 2 * self.num_kv_heads * self.block_tokens * self.head_dim * self.elem_bytes

    @property
    def block_bytes(self) -> int:
        return self.num_layers * self.tile_bytes


class _CacheC(C.Structure):
    _fields_ = [("d_pool", C.c_void_p), ("d_scales", C.c_void_p), ("layout", KVLayout),
                ("type", C.c_int32), ("inner", C.c_int32), ("layer", C.c_int32)]


class _BatchC(C.Structure):
    _fields_ = [("d_block_table", C.c_void_p), ("d_blk_off", C.c_void_p),
                ("table_stride", C.c_int64), ("d_tok_off", C.c_void_p), ("d_kv_len", C.c_void_p),
                ("n_tokens", C.c_int64), ("R", C.c_int32), ("max_new", C.c_int32)]


class _AttnC(C.Structure):
    _fields_ = [("q_type", C.c_int32), ("num_q_heads", C.c_int32), ("q_token_stride", C.c_int64),
                ("q_head_stride", C.c_int64), ("out_token_stride", C.c_int64),
                ("out_head_stride", C.c_int64), ("scale", C.c_float), ("causal", C.c_int32),
                ("window", C.c_int32)]


# The same three structures as bytes: a call passes what struct packs (0.3 us) instead of filling a
# ctypes object (1 us).
_CACHE_BYTES = struct.Struct("@PP6iI3i")
_BATCH_BYTES = struct.Struct("@PPqPPqii")
_ATTN_BYTES = struct.Struct("@iiqqqqfii")
_ROPE_BYTES = struct.Struct("@PPiif")
_ROPE_ROWS_BYTES = struct.Struct("@PPPP8qii")
_TABLES_BYTES = struct.Struct("@PPPqPPPPPqPPPPPPqiI")


class PodMetrics(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("d_throughput", "d_requests", "d_kv_usage",
                                          "d_queue_latency", "d_serve_latency")]


POLICY_RANDOM, POLICY_THROUGHPUT, POLICY_LEAST_REQUEST, POLICY_LEAST_KV_CACHE, \
    POLICY_LEAST_LATENCY, POLICY_PREFIX_CACHE_AWARE = range(6)

_lib = None


def lib():
    """The loaded C library.  Raises if it was never built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libaibx.so is missing at %s: build it with "
                "`python -m paper_2504_03648_b200.build` (needs nvcc, sm_100a)" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u32, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_uint64
        sig = {
            "aibx_hash_blocks": [vp, vp, vp, i32, i32, u64, vp, vp],
            "aibx_index_create": [C.POINTER(vp), u64, i32],
            "aibx_index_destroy": [vp],
            "aibx_index_clear": [vp, vp],
            "aibx_index_insert": [vp, vp, vp, vp, i64, vp],
            "aibx_index_evict": [vp, vp, vp, vp, i64, vp],
            "aibx_index_lookup": [vp, vp, vp, vp, i64, vp],
            "aibx_index_stats": [vp, C.POINTER(u64), C.POINTER(u64), vp],
            "aibx_index_stats2": [vp, C.POINTER(u64), C.POINTER(u64), C.POINTER(u64),
                                  C.POINTER(u32), vp],
            "aibx_index_touch": [vp, vp, i64, u32, vp],
            "aibx_index_pick_victims": [vp, u64, vp, vp, vp, vp],
            "aibx_index_export": [vp, vp, vp, vp, u64, vp, vp],
            "aibx_index_rehash": [vp, u64],
            "aibx_index_rehash_begin": [vp, u64, vp],
            "aibx_index_rehash_finish": [vp],
            "aibx_match_prefix": [vp, vp, vp, i32, vp, vp, vp, vp],
            "aibx_route_score": [vp, vp, i32, i32, vp, u64, C.POINTER(RouteParams), vp, vp, vp, vp],
            "aibx_route_batch": [vp, vp, vp, vp, i32, i32, u64, vp, u64, C.POINTER(RouteParams),
                                 vp, vp, vp, vp, vp, vp, vp],
            "aibx_route_assign": [vp, vp, i32, i32, vp, u64, C.POINTER(RouteParams), i32, vp, vp, vp],
            "aibx_route_head": [vp, vp, vp, vp, i32, i32, u64, vp, u64, C.POINTER(RouteParams),
                                vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "aibx_route_head_touch": [vp, vp, vp, vp, i32, i32, u64, vp, u64, C.POINTER(RouteParams),
                                      u32, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "aibx_route_head_collect": [vp, vp, vp, vp, i32, i32, u64, vp, u64, C.POINTER(RouteParams),
                                        u32, vp, vp, vp, vp, vp, vp, vp, vp, u32, vp, vp, vp, vp],
            "aibx_match_prefix_touch": [vp, vp, vp, i32, u32, vp, vp, vp, vp],
            "aibx_hash_blocks_resume": [vp, vp, vp, i32, i32, vp, vp, vp, vp],
            "aibx_route_policy": [i32, vp, vp, i32, i32, C.POINTER(PodMetrics), vp, u64, i32, vp, vp],
            "aibx_collect_blocks": [vp, i64, u32, vp, vp, vp, vp],
            "aibx_collect_blocks_static": [vp, i64, u32, vp, vp, vp],
            "aibx_kv_gather": [vp, C.POINTER(KVLayout), vp, i64, vp, vp],
            "aibx_kv_scatter": [vp, C.POINTER(KVLayout), vp, i64, vp, vp],
            "aibx_kv_gather_to_host": [vp, C.POINTER(KVLayout), vp, i64, vp, vp, vp],
            "aibx_kv_scatter_from_host": [vp, C.POINTER(KVLayout), vp, i64, vp, vp, vp],
            "aibx_kv_gather_counted": [vp, C.POINTER(KVLayout), vp, i64, vp, vp, vp],
            "aibx_kv_scatter_counted": [vp, C.POINTER(KVLayout), vp, i64, vp, vp, vp],
            "aibx_kv_gather_inner": [vp, C.POINTER(KVLayout), i32, i32, vp, i64, vp, vp],
            "aibx_kv_scatter_inner": [vp, C.POINTER(KVLayout), i32, i32, vp, i64, vp, vp],
            "aibx_kv_append": [vp, vp, vp, i64, i64, vp, i64, i64, i32, vp],
            "aibx_kv_read": [vp, vp, vp, i64, i64, vp, i64, i64, i32, vp],
            "aibx_attn_paged": [vp, vp, vp, vp, vp, vp, vp, u64, vp],
            "aibx_attn_tree": [vp, vp, vp, vp, i32, vp, vp, vp, vp, u64, vp],
            "aibx_tree_masks": [vp, vp, vp, i32, i64, i32, vp, vp, vp],
            "aibx_rope": [vp, i64, i32, i32, vp, i64, i64, vp, i64, i64, i32, vp],
            "aibx_rope_append": [vp, vp, vp, vp, vp],
            "aibx_kv_tables": [vp, i32, vp],
            "aibx_kv_set_tuning": [i32, i32, i32, i32],
            "aibx_kv_set_store_lag": [i32],
            "aibx_kv_get_tuning": [vp, vp, vp, vp, vp],
            "aibx_kv_set_inner_engine": [i32],
            "aibx_selftest_bounded_wait": [u32, vp],
            "aibx_status_fetch": [vp, C.POINTER(i32), C.POINTER(i64)],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = i32
        L.aibx_attn_workspace_bytes.argtypes = [vp, vp, vp]
        L.aibx_attn_workspace_bytes.restype = u64
        L.aibx_attn_tree_workspace_bytes.argtypes = [vp, vp, vp]
        L.aibx_attn_tree_workspace_bytes.restype = u64
        L.aibx_collect_scratch_bytes.argtypes = [u32]
        L.aibx_collect_scratch_bytes.restype = u64
        L.aibx_route_collect_scratch_bytes.argtypes = [u32]
        L.aibx_route_collect_scratch_bytes.restype = u64
        L.aibx_collect_static_max_blocks.argtypes = []
        L.aibx_collect_static_max_blocks.restype = u32
        L.aibx_strerror.argtypes = [i32]
        L.aibx_strerror.restype = C.c_char_p
        _lib = L
    return _lib


def _stream() -> int:
    # the handle itself: a torch Stream object around it costs as much as a launch (3 us)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t, dtype=None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensor expected"
    if dtype is not None:
        assert t.dtype == dtype, (t.dtype, dtype)
    return t.data_ptr()


def _check(call: str, rc: int) -> int:
    if rc != OK:
        raise AibxError(call, rc)
    return rc


def strerror(code: int) -> str:
    return lib().aibx_strerror(code).decode()


def hash_blocks(tokens, tok_off, blk_off, block_tokens: int, root_seed: int, hashes) -> None:
    R = tok_off.numel() - 1
    _check("aibx_hash_blocks", lib().aibx_hash_blocks(
        _ptr(tokens, torch.int32), _ptr(tok_off, torch.int64), _ptr(blk_off, torch.int64), R,
        block_tokens, root_seed & (2**64 - 1), _ptr(hashes, torch.uint64), _stream()))


class Index:
    """Host handle of a device-resident index (aibx_index_t)."""

    def __init__(self, capacity_slots: int, num_pods: int):
        h = C.c_void_p()
        self._h = None
        _check("aibx_index_create", lib().aibx_index_create(C.byref(h), capacity_slots, num_pods))
        self._h = h
        self.capacity = capacity_slots
        self.num_pods = num_pods

    def destroy(self) -> None:
        if self._h is not None:
            lib().aibx_index_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def clear(self) -> None:
        _check("aibx_index_clear", lib().aibx_index_clear(self._h, _stream()))

    def insert(self, keys, pod_masks, block_ids) -> None:
        n = keys.numel()
        _check("aibx_index_insert", lib().aibx_index_insert(
            self._h, _ptr(keys, torch.uint64), _ptr(pod_masks, torch.uint64),
            _ptr(block_ids, torch.uint32), n, _stream()))

    def evict(self, keys, pod_masks, freed_block_ids=None) -> None:
        n = keys.numel()
        _check("aibx_index_evict", lib().aibx_index_evict(
            self._h, _ptr(keys, torch.uint64), _ptr(pod_masks, torch.uint64),
            _ptr(freed_block_ids, torch.uint32), n, _stream()))

    def lookup(self, keys, masks=None, block_ids=None) -> None:
        n = keys.numel()
        _check("aibx_index_lookup", lib().aibx_index_lookup(
            self._h, _ptr(keys, torch.uint64), _ptr(masks, torch.uint64),
            _ptr(block_ids, torch.uint32), n, _stream()))

    def stats(self):
        live, cap = C.c_uint64(), C.c_uint64()
        _check("aibx_index_stats",
               lib().aibx_index_stats(self._h, C.byref(live), C.byref(cap), _stream()))
        return live.value, cap.value

    def stats2(self):
        """(live, removed, capacity, longest_walk)."""
        live, removed, cap, walk = C.c_uint64(), C.c_uint64(), C.c_uint64(), C.c_uint32()
        _check("aibx_index_stats2", lib().aibx_index_stats2(
            self._h, C.byref(live), C.byref(removed), C.byref(cap), C.byref(walk), _stream()))
        return live.value, removed.value, cap.value, walk.value

    def touch(self, keys, epoch: int) -> None:
        _check("aibx_index_touch", lib().aibx_index_touch(
            self._h, _ptr(keys, torch.uint64), keys.numel(), epoch, _stream()))

    def pick_victims(self, k: int, keys, priorities, count) -> None:
        _check("aibx_index_pick_victims", lib().aibx_index_pick_victims(
            self._h, k, _ptr(keys, torch.uint64), _ptr(priorities, torch.uint32),
            _ptr(count, torch.uint64), _stream()))

    def export(self, keys, masks, block_ids, count) -> None:
        """Live entries into the given arrays (any of them may be None); count: uint64[1]."""
        cap = min(t.numel() for t in (keys, masks, block_ids) if t is not None) \
            if any(t is not None for t in (keys, masks, block_ids)) else 0
        _check("aibx_index_export", lib().aibx_index_export(
            self._h, _ptr(keys, torch.uint64), _ptr(masks, torch.uint64),
            _ptr(block_ids, torch.uint32), cap, _ptr(count, torch.uint64), _stream()))

    def rehash(self, new_capacity: int) -> None:
        _check("aibx_index_rehash", lib().aibx_index_rehash(self._h, new_capacity))
        self.capacity = new_capacity

    def rehash_begin(self, new_capacity: int) -> None:
        """Start moving the index into a table of another size on the current stream; readers
        keep working on the old table until rehash_finish()."""
        _check("aibx_index_rehash_begin",
               lib().aibx_index_rehash_begin(self._h, new_capacity, _stream()))
        self._pending_capacity = new_capacity

    def rehash_finish(self) -> None:
        _check("aibx_index_rehash_finish", lib().aibx_index_rehash_finish(self._h))
        self.capacity = self._pending_capacity

    def match_prefix(self, hashes, blk_off, match_len, any_len=None, block_ids=None) -> None:
        R = blk_off.numel() - 1
        _check("aibx_match_prefix", lib().aibx_match_prefix(
            self._h, _ptr(hashes, torch.uint64), _ptr(blk_off, torch.int64), R,
            _ptr(match_len, torch.uint32), _ptr(any_len, torch.uint32),
            _ptr(block_ids, torch.uint32), _stream()))

    def match_prefix_touch(self, hashes, blk_off, epoch: int, match_len, any_len=None,
                           block_ids=None) -> None:
        """match_prefix that also marks the entries of every matched prefix as used in `epoch`."""
        R = blk_off.numel() - 1
        _check("aibx_match_prefix_touch", lib().aibx_match_prefix_touch(
            self._h, _ptr(hashes, torch.uint64), _ptr(blk_off, torch.int64), R, epoch,
            _ptr(match_len, torch.uint32), _ptr(any_len, torch.uint32),
            _ptr(block_ids, torch.uint32), _stream()))


def route_score(match_len, blk_off, num_pods: int, pod_load, ready_mask: int, params,
                best_pod, best_score, scores=None) -> None:
    R = blk_off.numel() - 1
    prm = None if params is None else C.byref(RouteParams(*params))
    _check("aibx_route_score", lib().aibx_route_score(
        _ptr(match_len, torch.uint32), _ptr(blk_off, torch.int64), R, num_pods,
        _ptr(pod_load, torch.int32), ready_mask & (2**64 - 1), prm, _ptr(best_pod, torch.int32),
        _ptr(best_score, torch.int64), _ptr(scores, torch.int64), _stream()))


def route_batch(index: Index, tokens, tok_off, blk_off, block_tokens: int, root_seed: int,
                pod_load, ready_mask: int, params, hashes, match_len, any_len, block_ids,
                best_pod, best_score) -> None:
    R = tok_off.numel() - 1
    prm = None if params is None else C.byref(RouteParams(*params))
    _check("aibx_route_batch", lib().aibx_route_batch(
        index._h, _ptr(tokens, torch.int32), _ptr(tok_off, torch.int64), _ptr(blk_off, torch.int64),
        R, block_tokens, root_seed & (2**64 - 1), _ptr(pod_load, torch.int32),
        ready_mask & (2**64 - 1), prm, _ptr(hashes, torch.uint64), _ptr(match_len, torch.uint32),
        _ptr(any_len, torch.uint32), _ptr(block_ids, torch.uint32), _ptr(best_pod, torch.int32),
        _ptr(best_score, torch.int64), _stream()))


def route_head(index: Index, tokens, tok_off, blk_off, block_tokens: int, root_seed: int,
               pod_load, ready_mask: int, params, hashes, match_len, any_len, block_ids,
               best_pod, best_score, hashed, next_seed) -> None:
    """Hash only as far as matching needs, match and score; `hashed`/`next_seed` receive the
    state hash_blocks_resume continues from."""
    R = tok_off.numel() - 1
    prm = None if params is None else C.byref(RouteParams(*params))
    _check("aibx_route_head", lib().aibx_route_head(
        index._h, _ptr(tokens, torch.int32), _ptr(tok_off, torch.int64), _ptr(blk_off, torch.int64),
        R, block_tokens, root_seed & (2**64 - 1), _ptr(pod_load, torch.int32),
        ready_mask & (2**64 - 1), prm, _ptr(hashes, torch.uint64), _ptr(match_len, torch.uint32),
        _ptr(any_len, torch.uint32), _ptr(block_ids, torch.uint32), _ptr(best_pod, torch.int32),
        _ptr(best_score, torch.int64), _ptr(hashed, torch.uint32), _ptr(next_seed, torch.uint64),
        _stream()))


def route_head_touch(index: Index, tokens, tok_off, blk_off, block_tokens: int, root_seed: int,
                     pod_load, ready_mask: int, params, epoch: int, hashes, match_len, any_len,
                     block_ids, best_pod, best_score, hashed, next_seed) -> None:
    """route_head that also marks the entries of every matched prefix as used in `epoch`."""
    R = tok_off.numel() - 1
    prm = None if params is None else C.byref(RouteParams(*params))
    _check("aibx_route_head_touch", lib().aibx_route_head_touch(
        index._h, _ptr(tokens, torch.int32), _ptr(tok_off, torch.int64), _ptr(blk_off, torch.int64),
        R, block_tokens, root_seed & (2**64 - 1), _ptr(pod_load, torch.int32),
        ready_mask & (2**64 - 1), prm, epoch, _ptr(hashes, torch.uint64),
        _ptr(match_len, torch.uint32), _ptr(any_len, torch.uint32), _ptr(block_ids, torch.uint32),
        _ptr(best_pod, torch.int32), _ptr(best_score, torch.int64), _ptr(hashed, torch.uint32),
        _ptr(next_seed, torch.uint64), _stream()))


def route_collect_scratch_bytes(num_blocks: int) -> int:
    return int(lib().aibx_route_collect_scratch_bytes(num_blocks))


def route_head_collect(index: Index, tokens, tok_off, blk_off, block_tokens: int, root_seed: int,
                       pod_load, ready_mask: int, params, epoch: int, hashes, match_len, any_len,
                       block_ids, best_pod, best_score, hashed, next_seed, num_blocks: int,
                       scratch, unique_ids, count) -> None:
    """route_head (+ stamping when epoch > 0) that also leaves the set of matched blocks in
    unique_ids / count, without a further launch."""
    R = tok_off.numel() - 1
    prm = None if params is None else C.byref(RouteParams(*params))
    _check("aibx_route_head_collect", lib().aibx_route_head_collect(
        index._h, _ptr(tokens, torch.int32), _ptr(tok_off, torch.int64), _ptr(blk_off, torch.int64),
        R, block_tokens, root_seed & (2**64 - 1), _ptr(pod_load, torch.int32),
        ready_mask & (2**64 - 1), prm, epoch, _ptr(hashes, torch.uint64),
        _ptr(match_len, torch.uint32), _ptr(any_len, torch.uint32), _ptr(block_ids, torch.uint32),
        _ptr(best_pod, torch.int32), _ptr(best_score, torch.int64), _ptr(hashed, torch.uint32),
        _ptr(next_seed, torch.uint64), num_blocks, _ptr(scratch), _ptr(unique_ids, torch.uint32),
        _ptr(count, torch.uint32), _stream()))


def hash_blocks_resume(tokens, tok_off, blk_off, block_tokens: int, hashed, next_seed,
                       hashes) -> None:
    R = tok_off.numel() - 1
    _check("aibx_hash_blocks_resume", lib().aibx_hash_blocks_resume(
        _ptr(tokens, torch.int32), _ptr(tok_off, torch.int64), _ptr(blk_off, torch.int64), R,
        block_tokens, _ptr(hashed, torch.uint32), _ptr(next_seed, torch.uint64),
        _ptr(hashes, torch.uint64), _stream()))


def route_assign(match_len, blk_off, num_pods: int, pod_load, ready_mask: int, params,
                 load_increment: int, best_pod, best_score) -> None:
    R = blk_off.numel() - 1
    prm = None if params is None else C.byref(RouteParams(*params))
    _check("aibx_route_assign", lib().aibx_route_assign(
        _ptr(match_len, torch.uint32), _ptr(blk_off, torch.int64), R, num_pods,
        _ptr(pod_load, torch.int32), ready_mask & (2**64 - 1), prm, load_increment,
        _ptr(best_pod, torch.int32), _ptr(best_score, torch.int64), _stream()))


def route_policy(policy: int, num_pods: int, R: int, ready_mask: int, best_pod, throughput=None,
                 requests=None, kv_usage=None, queue_latency=None, serve_latency=None,
                 match_len=None, blk_off=None, draws=None, threshold_pct: int = 50) -> None:
    """One pod per request under one of the six policies (POLICY_* numbers); the per-pod
    figures are int32 device tensors, only those the policy reads are needed."""
    figs = (throughput, requests, kv_usage, queue_latency, serve_latency)
    met = None
    if any(t is not None for t in figs):
        met = C.byref(PodMetrics(*[_ptr(t, torch.int32) for t in figs]))
    _check("aibx_route_policy", lib().aibx_route_policy(
        policy, _ptr(match_len, torch.uint32), _ptr(blk_off, torch.int64), R, num_pods, met,
        _ptr(draws, torch.uint64), ready_mask & (2**64 - 1), threshold_pct,
        _ptr(best_pod, torch.int32), _stream()))


def collect_scratch_bytes(num_blocks: int) -> int:
    return int(lib().aibx_collect_scratch_bytes(num_blocks))


def collect_blocks(block_ids, num_blocks: int, scratch, unique_ids, count) -> None:
    n = block_ids.numel()
    assert scratch.numel() * scratch.element_size() >= collect_scratch_bytes(num_blocks)
    assert unique_ids.numel() >= n
    _check("aibx_collect_blocks", lib().aibx_collect_blocks(
        _ptr(block_ids, torch.uint32), n, num_blocks, _ptr(scratch), _ptr(unique_ids, torch.uint32),
        _ptr(count, torch.uint32), _stream()))


def collect_static_max_blocks() -> int:
    return int(lib().aibx_collect_static_max_blocks())


def collect_blocks_static(block_ids, num_blocks: int, unique_ids, count) -> None:
    """collect_blocks for callers that must not allocate: the bitmap is the library's own fixed
    array (pools up to collect_static_max_blocks() blocks).  Calls on one device share that
    array, so they must not overlap on the GPU."""
    n = block_ids.numel()
    assert unique_ids.numel() >= n
    _check("aibx_collect_blocks_static", lib().aibx_collect_blocks_static(
        _ptr(block_ids, torch.uint32), n, num_blocks, _ptr(unique_ids, torch.uint32),
        _ptr(count, torch.uint32), _stream()))


def kv_gather(pool, layout: KVLayout, block_ids, n: int, buf) -> None:
    _check("aibx_kv_gather", lib().aibx_kv_gather(
        _ptr(pool), C.byref(layout), _ptr(block_ids, torch.uint32), n, _ptr(buf), _stream()))


def kv_scatter(pool, layout: KVLayout, block_ids, n: int, buf) -> None:
    _check("aibx_kv_scatter", lib().aibx_kv_scatter(
        _ptr(pool), C.byref(layout), _ptr(block_ids, torch.uint32), n, _ptr(buf), _stream()))


def kv_gather_to_host(pool, layout: KVLayout, block_ids, n: int, staging, host_buf) -> None:
    """Gather into the device staging buffer, then on to `host_buf` (a CPU tensor, pinned for an
    asynchronous copy), all on the current stream."""
    assert not host_buf.is_cuda and host_buf.is_contiguous()
    _check("aibx_kv_gather_to_host", lib().aibx_kv_gather_to_host(
        _ptr(pool), C.byref(layout), _ptr(block_ids, torch.uint32), n, _ptr(staging),
        host_buf.data_ptr(), _stream()))


def kv_scatter_from_host(pool, layout: KVLayout, block_ids, n: int, staging, host_buf) -> None:
    """`host_buf` (CPU tensor) into the device staging buffer, then scatter, on the current stream."""
    assert not host_buf.is_cuda and host_buf.is_contiguous()
    _check("aibx_kv_scatter_from_host", lib().aibx_kv_scatter_from_host(
        _ptr(pool), C.byref(layout), _ptr(block_ids, torch.uint32), n, _ptr(staging),
        host_buf.data_ptr(), _stream()))


def kv_gather_counted(pool, layout: KVLayout, block_ids, n_max: int, count, buf) -> None:
    _check("aibx_kv_gather_counted", lib().aibx_kv_gather_counted(
        _ptr(pool), C.byref(layout), _ptr(block_ids, torch.uint32), n_max,
        _ptr(count, torch.uint32), _ptr(buf), _stream()))


def kv_scatter_counted(pool, layout: KVLayout, block_ids, n_max: int, count, buf) -> None:
    _check("aibx_kv_scatter_counted", lib().aibx_kv_scatter_counted(
        _ptr(pool), C.byref(layout), _ptr(block_ids, torch.uint32), n_max,
        _ptr(count, torch.uint32), _ptr(buf), _stream()))


def kv_gather_inner(pool, layout: KVLayout, pool_inner: int, buf_inner: int, block_ids, n: int,
                    buf) -> None:
    _check("aibx_kv_gather_inner", lib().aibx_kv_gather_inner(
        _ptr(pool), C.byref(layout), pool_inner, buf_inner, _ptr(block_ids, torch.uint32), n,
        _ptr(buf), _stream()))


def kv_scatter_inner(pool, layout: KVLayout, pool_inner: int, buf_inner: int, block_ids, n: int,
                     buf) -> None:
    _check("aibx_kv_scatter_inner", lib().aibx_kv_scatter_inner(
        _ptr(pool), C.byref(layout), pool_inner, buf_inner, _ptr(block_ids, torch.uint32), n,
        _ptr(buf), _stream()))


class KVCache:
    """One layer of a paged pool whose rows have a type (aibx_kv_cache_t).  `pool` is the pool as
    kv_gather takes it (any dtype), `scales` the byte pool of an e4m3 one.  Setting `layer` moves
    the view to another layer."""

    def __init__(self, pool, layout: KVLayout, type: int, scales=None, inner: int = 0,
                 layer: int = 0):
        self._keep = (pool, scales)
        self.device = pool.get_device()
        self.layout = layout
        kind, layers, heads, slots, dim, size, blocks = (
            layout.layout, layout.num_layers, layout.num_kv_heads, layout.block_tokens, layout.head_dim,
            layout.elem_bytes, layout.num_blocks)
        self.heads, self.head_dim = heads, dim
        # a pool that is smaller than its layout says is a fault waiting to happen
        rows = blocks * layers * 2 * heads * slots
        if pool.nbytes < rows * dim * size:
            raise ValueError("pool of %d bytes, layout of %d rows of %d elements of %d bytes" % (
                pool.nbytes, rows, dim, size))
        if scales is not None and (scales.get_device() != self.device or scales.numel() < rows):
            raise ValueError("%d scale bytes on the pool's device expected" % rows)
        self._fields = [_ptr(pool), 0 if scales is None else _ptr(scales, torch.uint8), kind, layers, heads, slots,
                        dim, size, blocks, type, inner, layer]
        self._ref = _CACHE_BYTES.pack(*self._fields)

    @property
    def layer(self) -> int:
        return self._fields[-1]

    @layer.setter
    def layer(self, n: int) -> None:
        self._fields[-1] = n
        self._ref = _CACHE_BYTES.pack(*self._fields)


class KVBatch:
    """Which tokens of which requests a call is about (aibx_kv_batch_t): the last
    tok_off[r+1] - tok_off[r] of request r's kv_len[r] tokens.  block_table: uint32 [R, width], or
    flat with blk_off (int64 [R+1]).  n_tokens: rows of the per-token tensors.  max_new: a bound on
    the tokens of one request, if known."""

    def __init__(self, block_table, tok_off, kv_len, n_tokens: int, max_new: int = 0, blk_off=None):
        R = kv_len.numel()
        if tok_off.numel() != R + 1 or (blk_off is not None and blk_off.numel() != R + 1):
            raise ValueError("offsets of %d requests expected" % R)
        if blk_off is None and (block_table.dim() != 2 or block_table.shape[0] != R):
            raise ValueError("a block table of %d rows expected" % R)
        self._keep = (block_table, tok_off, kv_len, blk_off)
        self.device = kv_len.get_device()
        if block_table.get_device() != self.device or tok_off.get_device() != self.device or \
                (blk_off is not None and blk_off.get_device() != self.device):
            raise ValueError("all tensors of a batch live on one CUDA device")
        self.n_tokens = n_tokens
        self._ref = _BATCH_BYTES.pack(
            _ptr(block_table, torch.uint32), 0 if blk_off is None else _ptr(blk_off, torch.int64),
            0 if blk_off is not None else block_table.shape[1], _ptr(tok_off, torch.int64),
            _ptr(kv_len, torch.int32), n_tokens, R, max_new)


def _rows(t, cache: KVCache, batch: KVBatch, heads: int):
    """(pointer, token stride, head stride) of a [n_tokens, heads, head_dim] tensor."""
    n, h, d = t.shape
    st = t.stride()
    if n != batch.n_tokens or h != heads or d != cache.head_dim or (st[2] != 1 and d > 1):
        raise ValueError("rows of [%d, %d, %d] expected, got %s with strides %s" % (
            batch.n_tokens, heads, cache.head_dim, tuple(t.shape), st))
    if t.get_device() != cache.device:
        raise ValueError("all tensors of a call live on one CUDA device")
    return t.data_ptr(), st[0], st[1]


def _here(cache: KVCache, batch: KVBatch) -> int:
    """The current stream, once it is sure that everything lives on the current device."""
    if cache.device != batch.device or cache.device != torch._C._cuda_getDevice():
        raise ValueError("the call works on the current device (%d); pool on %d, batch on %d" % (
            torch._C._cuda_getDevice(), cache.device, batch.device))
    return torch._C._cuda_getCurrentRawStream(cache.device)


def _kv_tokens(name: str, cache: KVCache, batch: KVBatch, k, v) -> None:
    if k.dtype != v.dtype or k.dtype not in _TYPE_OF:
        raise ValueError("K and V of one of bfloat16, float16, float32 expected")
    stream = _here(cache, batch)
    kp, kt, kh = _rows(k, cache, batch, cache.heads)
    vp, vt, vh = _rows(v, cache, batch, cache.heads)
    _check(name, getattr(lib(), name)(cache._ref, batch._ref, kp, kt, kh, vp, vt, vh,
                                      _TYPE_OF[k.dtype], stream))


def kv_append(cache: KVCache, batch: KVBatch, k, v) -> None:
    """Write the batch's tokens (k, v: [n_tokens, kv_heads, head_dim], rows adjacent, other strides
    free) into their slots, quantised where the pool is e4m3."""
    _kv_tokens("aibx_kv_append", cache, batch, k, v)


def kv_read(cache: KVCache, batch: KVBatch, k, v) -> None:
    """Read the batch's tokens back into k, v (bfloat16, float16 or float32)."""
    _kv_tokens("aibx_kv_read", cache, batch, k, v)


def _attention(name: str, cache: KVCache, batch: KVBatch, tree, q, out, lse, scale, causal, window,
               workspace) -> None:
    if q.dtype != out.dtype or q.dtype not in _TYPE_OF or q.dim() != 3:
        raise ValueError("queries and output of one type and [n_tokens, q_heads, head_dim] expected")
    stream = _here(cache, batch)
    heads = q.shape[1]
    qp, qt, qh = _rows(q, cache, batch, heads)
    op, ot, oh = _rows(out, cache, batch, heads)
    lp = None
    if lse is not None:
        if lse.numel() != batch.n_tokens * heads or lse.dim() != 2 or lse.shape[1] != heads or lse.dtype != torch.float32 or not lse.is_contiguous() or \
                lse.get_device() != cache.device:
            raise ValueError("lse of float32 [n_tokens, q_heads], contiguous, expected")
        lp = lse.data_ptr()
    ref = _ATTN_BYTES.pack(_TYPE_OF[q.dtype], heads, qt, qh, ot, oh,
                           cache.head_dim ** -0.5 if scale is None else scale, 1 if causal else 0, window)
    L = lib()
    if workspace is None:
        size = L.aibx_attn_tree_workspace_bytes if tree else L.aibx_attn_workspace_bytes
        workspace = q.new_empty(max(size(cache._ref, batch._ref, ref), 16), dtype=torch.uint8)
    elif workspace.get_device() != cache.device or not workspace.is_contiguous():
        raise ValueError("a contiguous workspace on the pool's device expected")
    _check(name, getattr(L, name)(cache._ref, batch._ref, ref, *tree, qp, op, lp, workspace.data_ptr(),
                                  workspace.nbytes, stream))


def attn_paged(cache: KVCache, batch: KVBatch, q, out, lse=None, scale=None, causal: bool = True,
               window: int = 0, workspace=None) -> None:
    """Attention of the batch's tokens over their requests' cached keys.  q, out: [n_tokens,
    q_heads, head_dim]; lse: float32 [n_tokens, q_heads] or None; scale: 1/sqrt(head_dim) if None.
    workspace: uint8 tensor of attn_workspace_bytes(...) bytes, allocated here if None."""
    _attention("aibx_attn_paged", cache, batch, (), q, out, lse, scale, causal, window, workspace)


def _vector(t, what: str, dtype, n: int, device: int) -> int:
    """Pointer of n contiguous numbers of a type, on the call's device."""
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        raise ValueError("%s: %d contiguous numbers of %s on device %d expected, got %s of %s on %s" % (
            what, n, dtype, device, tuple(t.shape), t.dtype, t.device))
    return t.data_ptr()


def _current(t) -> int:
    """The current device, which a call's tensors live on."""
    device = torch._C._cuda_getDevice()
    if t.get_device() != device:
        raise ValueError("the call works on the current device (%d), not on %s" % (device, t.device))
    return device


def tree_masks(parent, tok_off, kv_len, mask, pos=None) -> None:
    """What each node of the requests' drafted trees sees: parent int32 [n_tokens] (index in the
    request, negative: none) -> mask uint64 [n_tokens, words], and pos int32 [n_tokens] (its position
    in the text).  kv_len is read for pos alone, and may be None without it."""
    device = _current(parent)
    n, R = parent.numel(), tok_off.numel() - 1
    if mask.dim() != 2 or mask.shape[0] != n or R < 0:
        raise ValueError("a mask of %d rows and offsets of every request expected" % n)
    words = mask.shape[1]
    _check("aibx_tree_masks", lib().aibx_tree_masks(
        _vector(parent, "parent", torch.int32, n, device), _vector(tok_off, "tok_off", torch.int64, R + 1, device),
        None if kv_len is None else _vector(kv_len, "kv_len", torch.int32, R, device), R, n, words,
        _vector(mask, "mask", torch.uint64, n * words, device),
        None if pos is None else _vector(pos, "pos", torch.int32, n, device),
        torch._C._cuda_getCurrentRawStream(device)))


def attn_tree(cache: KVCache, batch: KVBatch, mask, q, out, lse=None, scale=None, window: int = 0,
              workspace=None) -> None:
    """attn_paged of drafted tokens that see their request's cached tokens and the drafted ones that
    mask (uint64 [n_tokens, words], as tree_masks makes it) names.  The window hides cached tokens alone: with
    the bits of ancestors `window` and more nodes up cleared, a chain sees what attn_paged would show it."""
    if mask.dim() != 2:
        raise ValueError("a mask of [n_tokens, words] expected")
    tree = _vector(mask, "mask", torch.uint64, batch.n_tokens * mask.shape[1], cache.device), mask.shape[1]
    _attention("aibx_attn_tree", cache, batch, tree, q, out, lse, scale, False, window, workspace)


class Rope:
    """Rotary positions (aibx_rope_t): inv_freq float64 [rotary_dim / 2] on the device, radians per
    position of each pair; factor on sine and cosine."""

    def __init__(self, inv_freq, interleaved: bool = False, factor: float = 1.0):
        self.device = inv_freq.get_device()
        self._keep = inv_freq
        self._fields = (_vector(inv_freq, "inv_freq", torch.float64, inv_freq.numel(), self.device),
                        2 * inv_freq.numel(), ROPE_INTERLEAVED if interleaved else ROPE_HALF, factor)

    def _pack(self, pos, n: int) -> bytes:
        p, dim, style, factor = self._fields
        return _ROPE_BYTES.pack(p, 0 if pos is None else _vector(pos, "pos", torch.int32, n, self.device), dim,
                                style, factor)


def rope_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none", scale: float = 1.0,
                     trained: int = 0, fast: float = 32.0, slow: float = 1.0):
    """(inv_freq, factor) for Rope, float64 on the host: base^(-2 i / rotary_dim) and 1, or scaled for
    contexts `scale` times as long as the trained one:
    "linear": every frequency over scale;
    "base":   base * scale^(rotary_dim / (rotary_dim - 2)), which stretches the slowest pair alone by scale;
    "parts":  pairs of at most `slow` turns over the `trained` positions over scale, pairs of `fast` turns
              or more as they are, between them a straight line in the number of turns (a line in the
              pair's index, which some programs draw, gives other frequencies there); factor
              0.1 ln(scale) + 1."""
    if rotary_dim <= 0 or rotary_dim % 2 or base <= 0 or scale <= 0:
        raise ValueError("an even positive rotary_dim, base and scale above 0 expected")
    half = rotary_dim // 2
    if scaling == "base":
        if rotary_dim == 2:
            raise ValueError("a single pair has no base to scale")
        base = base * scale ** (rotary_dim / (rotary_dim - 2))
    f = base ** (-torch.arange(half, dtype=torch.float64) / half)
    if scaling in ("none", "base"):
        return f, 1.0
    if scaling == "linear":
        return f / scale, 1.0
    if scaling != "parts":
        raise ValueError("scaling none, linear, base or parts expected, got %r" % scaling)
    if trained <= 0 or fast <= slow:
        raise ValueError("parts: trained positions and fast > slow expected")
    turns = trained * f / 6.283185307179586
    keep = ((turns - slow) / (fast - slow)).clamp(0, 1)
    log = torch.log(torch.tensor(max(scale, 1.0), dtype=torch.float64)).item()
    return f * (keep + (1 - keep) / scale), 0.1 * log + 1.0


def rope(rope: Rope, pos, x, y) -> None:
    """Rows of x ([n_tokens, heads, head_dim], elements adjacent, other strides free) turned by their
    positions (int32 [n_tokens]) into y; y may be x, and is no tensor expanded over tokens or heads."""
    if x.dtype != y.dtype or x.dtype not in _TYPE_OF or x.dim() != 3 or x.shape != y.shape:
        raise ValueError("x and y of one type and [n_tokens, heads, head_dim] expected")
    device = _current(x)
    xs, ys = x.stride(), y.stride()
    if (x.shape[2] > 1 and (xs[2] != 1 or ys[2] != 1)) or y.get_device() != device or rope.device != device:
        raise ValueError("rows of adjacent elements on one device expected")
    n, heads, dim = x.shape
    _check("aibx_rope", lib().aibx_rope(rope._pack(pos, n), n, heads, dim, x.data_ptr(), xs[0], xs[1], y.data_ptr(),
                                        ys[0], ys[1], _TYPE_OF[x.dtype],
                                        torch._C._cuda_getCurrentRawStream(device)))


def rope_append(cache: KVCache, batch: KVBatch, rope: Rope, k, v, q=None, q_out=None, pos=None) -> None:
    """kv_append of k turned by its positions and of v as it is; q ([n_tokens, q_heads, head_dim])
    turned into q_out (which may be q) beside them.  pos: int32 [n_tokens], or the batch's positions."""
    if k.dtype != v.dtype or k.dtype not in _TYPE_OF or (q is None) != (q_out is None):
        raise ValueError("K, V and queries of one of bfloat16, float16, float32 expected")
    stream = _here(cache, batch)
    if rope.device != cache.device:
        raise ValueError("all tensors of a call live on one CUDA device")
    kp, kt, kh = _rows(k, cache, batch, cache.heads)
    vp, vt, vh = _rows(v, cache, batch, cache.heads)
    heads = qp = qt = qh = op = ot = oh = 0
    if q is not None:
        if q.dtype != k.dtype or q_out.dtype != k.dtype or q.dim() != 3:
            raise ValueError("queries of K's type and [n_tokens, q_heads, head_dim] expected")
        heads = q.shape[1]
        qp, qt, qh = _rows(q, cache, batch, heads)
        op, ot, oh = _rows(q_out, cache, batch, heads)
    rows = _ROPE_ROWS_BYTES.pack(qp, op, kp, vp, qt, qh, ot, oh, kt, kh, vt, vh, heads, _TYPE_OF[k.dtype])
    _check("aibx_rope_append", lib().aibx_rope_append(cache._ref, batch._ref, rope._pack(pos, batch.n_tokens), rows,
                                                      stream))


def kv_tables(held, new, block_tokens: int, num_blocks: int, free_ids, head, tail, block_table, tok_off,
              kv_len, n_tokens: int, pos=None, slots=None, head_out=None, blk_off=None, match_ids=None,
              match_off=None) -> None:
    """Grows the requests' rows of block_table (uint32 [R, width], or flat with blk_off) from `held` to
    held + new tokens (int32 [R]) by ids of the free list (free_ids uint32, a ring; head, tail int64 [1]:
    numbers of the first id to take and of the first that is not there), and leaves tok_off (int64
    [R+1]), kv_len (int32 [R], may be `held`), pos (int32 [n_tokens]), slots (int64 [n_tokens]) and the
    new head (head_out, `head` itself if None).  match_ids (uint32) with match_off (int64 [R+1]): the
    blocks that hold the held tokens, copied into the rows."""
    device = _current(held)
    R = held.numel()
    if (match_ids is None) != (match_off is None):
        raise ValueError("match_ids and match_off come together")
    if blk_off is None and (block_table.dim() != 2 or block_table.shape[0] != R):
        raise ValueError("a block table of %d rows expected" % R)

    def vec(t, what, dtype, n):
        return 0 if t is None else _vector(t, what, dtype, n, device)

    ref = _TABLES_BYTES.pack(
        vec(held, "held", torch.int32, R), vec(new, "new", torch.int32, R),
        vec(free_ids, "free_ids", torch.uint32, free_ids.numel()), free_ids.numel(), vec(head, "head", torch.int64, 1),
        vec(tail, "tail", torch.int64, 1), vec(head if head_out is None else head_out, "head_out", torch.int64, 1),
        vec(block_table, "block_table", torch.uint32, block_table.numel()), vec(blk_off, "blk_off", torch.int64, R + 1),
        0 if blk_off is not None else block_table.shape[1],
        0 if match_ids is None else vec(match_ids, "match_ids", torch.uint32, match_ids.numel()),
        vec(match_off, "match_off", torch.int64, R + 1), vec(tok_off, "tok_off", torch.int64, R + 1),
        vec(kv_len, "kv_len", torch.int32, R), vec(pos, "pos", torch.int32, n_tokens),
        vec(slots, "slots", torch.int64, n_tokens), n_tokens, block_tokens, num_blocks)
    _check("aibx_kv_tables", lib().aibx_kv_tables(ref, R, torch._C._cuda_getCurrentRawStream(device)))


def _workspace_bytes(name: str, cache: KVCache, batch: KVBatch, q) -> int:
    return int(getattr(lib(), name)(cache._ref, batch._ref, _ATTN_BYTES.pack(
        _TYPE_OF.get(q.dtype, -1), q.shape[1], 8, 8, 8, 8, 1.0, 1, 0)))


def attn_workspace_bytes(cache: KVCache, batch: KVBatch, q) -> int:
    """Workspace of attn_paged for queries shaped like q; 0 where attn_paged would refuse."""
    return _workspace_bytes("aibx_attn_workspace_bytes", cache, batch, q)


def attn_tree_workspace_bytes(cache: KVCache, batch: KVBatch, q) -> int:
    """The same of attn_tree."""
    return _workspace_bytes("aibx_attn_tree_workspace_bytes", cache, batch, q)


def kv_set_tuning(mode: int = -1, chunk_bytes: int = 0, stages: int = 0,
                  ctas_per_sm: int = 0) -> None:
    _check("aibx_kv_set_tuning", lib().aibx_kv_set_tuning(mode, chunk_bytes, stages, ctas_per_sm))


def kv_get_tuning():
    """(mode, chunk_bytes, stages, ctas_per_sm, lag) as a copy call starting now would read them."""
    v = [C.c_int32() for _ in range(5)]
    _check("aibx_kv_get_tuning", lib().aibx_kv_get_tuning(*[C.addressof(x) for x in v]))
    return tuple(x.value for x in v)


def kv_set_inner_engine(engine: int = 0) -> None:
    """0 tensor-map store with fallback, 1 storer warps, 2 tensor-map store or UNSUPPORTED."""
    _check("aibx_kv_set_inner_engine", lib().aibx_kv_set_inner_engine(engine))


def kv_set_store_lag(lag: int = 1) -> None:
    _check("aibx_kv_set_store_lag", lib().aibx_kv_set_store_lag(lag))


def selftest_bounded_wait(spins: int = 1000) -> None:
    _check("aibx_selftest_bounded_wait", lib().aibx_selftest_bounded_wait(spins, _stream()))


def status_fetch():
    """(status, detail) of the current device since the last fetch; synchronises the stream."""
    st, det = C.c_int32(), C.c_int64()
    _check("aibx_status_fetch", lib().aibx_status_fetch(_stream(), C.byref(st), C.byref(det)))
    return st.value, det.value
