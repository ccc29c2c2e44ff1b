"""Python binding of libsmetric.so, the GB300 batched routing path of
balanced session-centric scheduling (SMetric, arXiv 2607.08565).

Functions carry the C ABI's names and only marshal arguments: device arrays
may be passed as torch tensors or raw device pointers (ints); streams as a
torch.cuda.Stream, a raw cudaStream_t (int) or None for torch's current
stream. Every computation runs in the library's CUDA kernels; there is no
CPU fallback, and using the binding without the built library raises.

SMetricIndex wraps one index, SMetricKV one handle of the paged KV$
operators and SMetricKV4 one with its caches in 4 bits; they allocate output
tensors for convenience.
"""

from __future__ import annotations

import ctypes as C
import os
from typing import Any, NamedTuple, Optional

from .build_lib import LIB as _LIB_PATH

SMETRIC_OK = 0
SMETRIC_ERR_INVALID_ARG = -1
SMETRIC_ERR_OOM = -2
SMETRIC_ERR_TABLE_FULL = -3
SMETRIC_ERR_CUDA = -4
SMETRIC_ERR_OVERFLOW = -5
SMETRIC_ERR_TOO_LARGE = -6
SMETRIC_NOALLOC_MAX_REQUESTS = 4096
SMETRIC_NOALLOC_MAX_BLOCKS = 32768
SMETRIC_MAX_INSTANCES = 256
SMETRIC_MAX_WEIGHT = 1 << 20
SMETRIC_MAX_LOAD = 1 << 40
SMETRIC_MAX_PROBE = 65536
SMETRIC_FLAG_HOST_STAGING = 1
SMETRIC_FLAG_PIPELINE = 2
SMETRIC_POLICY_MAX_LEN = 1 << 24
SMETRIC_POLICY_MAX_QUEUED = 1 << 59
SMETRIC_COMMIT_GLOBAL = 1
SMETRIC_POLICY_MAX_TPOT = 1 << 60
SMETRIC_POLICY_MAX_REQUESTS = 1 << 20
SMETRIC_IMBALANCE_MAX_WINDOW = 1 << 36
SMETRIC_IMBALANCE_MAX_REQUESTS = 1 << 26
SMETRIC_IMBALANCE_MAX_CELLS = 1 << 31
SMETRIC_SCORER_BAILIAN = 1
SMETRIC_SCORER_LMETRIC = 2
SMETRIC_BF16 = 0
SMETRIC_F16 = 1
SMETRIC_KV_MAX_HEAD_DIM = 128
SMETRIC_KV_MAX_GROUP = 128
SMETRIC_KV_MAX_REQUESTS = 1 << 20
SMETRIC_KV_MAX_TOKENS = 1 << 26
SMETRIC_KV_INTERLEAVED = 1
SMETRIC_KV_4BIT = 2
SMETRIC_KVQ_MAX_EXP = 64
SMETRIC_KVQ_MAX_ROWS = 1 << 30

EXPORTED = (
    "smetric_index_create", "smetric_index_destroy", "smetric_index_clear",
    "smetric_index_insert", "smetric_index_evict", "smetric_index_lookup",
    "smetric_index_mask_words", "smetric_route_batch", "smetric_block_hashes",
    "smetric_route_batch_host", "smetric_status", "smetric_strerror",
    "smetric_profile_enable", "smetric_profile_read", "smetric_profile_kernel_name",
    "smetric_launch_count", "smetric_block_hashes_noalloc", "smetric_route_batch_policy",
    "smetric_index_commit_batch", "smetric_route_batch_policy_coloc", "smetric_link_sessions",
    "smetric_route_batch_baseline", "smetric_route_batch_sequential", "smetric_reuse_workspace_bytes",
    "smetric_reuse_breakdown", "smetric_imbalance_workspace_bytes", "smetric_window_imbalance",
    "smetric_route_batches", "smetric_index_set_lru", "smetric_index_lru_sizes", "smetric_route_commit_batch",
    "smetric_kv_create", "smetric_kv_destroy", "smetric_kv_plan", "smetric_kv_append", "smetric_qk_norm_rope",
    "smetric_paged_attention", "smetric_kv_status", "smetric_kv_launch_count",
    "smetric_kvq_append", "smetric_kvq_read", "smetric_kvq_attention", "smetric_kv_plan_up_to",
)


class SmetricError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {smetric_strerror(code)} ({code})")


class smetric_index_config(C.Structure):
    _fields_ = [
        ("num_instances", C.c_int32),
        ("block_size", C.c_int32),
        ("session_blocks", C.c_int32),
        ("flags", C.c_int32),
        ("capacity_slots", C.c_uint64),
        ("hash_seed", C.c_uint64),
        ("max_batch_requests", C.c_int64),
        ("max_batch_tokens", C.c_int64),
    ]


class smetric_weights(C.Structure):
    _fields_ = [("w_load", C.c_int64), ("w_miss", C.c_int64), ("w_glob", C.c_int64)]


class smetric_policy(C.Structure):
    _fields_ = [("c_lin", C.c_int64), ("c_att", C.c_int64), ("ttft_d0", C.c_int64),
                ("ttft_d1", C.c_int64), ("hit_num", C.c_int64), ("hit_den", C.c_int64),
                ("rr_base", C.c_int32), ("reserved", C.c_int32)]


class smetric_kv_config(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
                ("page_size", C.c_int32), ("dtype", C.c_int32), ("flags", C.c_int32), ("num_pages", C.c_int64),
                ("max_batch_requests", C.c_int64), ("max_batch_tokens", C.c_int64)]


class smetric_heads(C.Structure):
    _fields_ = [("d_data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class smetric_kv_cache(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("page_stride", C.c_int64), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64)]


class smetric_kvq_cache(C.Structure):
    _fields_ = [("d_codes", C.c_void_p), ("d_scales", C.c_void_p), ("page_stride", C.c_int64), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64), ("scale_page_stride", C.c_int64), ("scale_token_stride", C.c_int64),
                ("scale_head_stride", C.c_int64), ("exp", C.c_int32), ("reserved", C.c_int32)]


class smetric_kv_transform(C.Structure):
    _fields_ = [("d_cos_sin", C.c_void_p), ("table_rows", C.c_int64), ("d_q_norm", C.c_void_p),
                ("d_k_norm", C.c_void_p), ("eps", C.c_float), ("rot_dim", C.c_int32), ("flags", C.c_int32),
                ("reserved", C.c_int32)]


_lib = None


def library_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded libsmetric.so. Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"libsmetric.so is not built ({_LIB_PATH}); run __graft_entry__.build() "
                "or python -m paper_2607_08565_gb300.build_lib")
        L = C.CDLL(_LIB_PATH)
        P, I32, I64, U64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
        sig = {
            "smetric_index_create": (C.c_int, [C.POINTER(smetric_index_config), C.POINTER(P)]),
            "smetric_index_destroy": (C.c_int, [P]),
            "smetric_index_clear": (C.c_int, [P, P]),
            "smetric_index_insert": (C.c_int, [P, P, P, I64, P]),
            "smetric_index_evict": (C.c_int, [P, P, P, I64, P]),
            "smetric_index_lookup": (C.c_int, [P, P, I64, P, P]),
            "smetric_index_mask_words": (I32, [P]),
            "smetric_route_batch": (C.c_int, [P, P, I64, P, I32, P, smetric_weights, P, P, P, P, P,
                                              I64, P]),
            "smetric_route_batches": (C.c_int, [P, I32, P, P, P, P, P, smetric_weights, P, P, P, P, P]),
            "smetric_route_batch_policy": (C.c_int, [P, P, I64, P, I32, P, P, P, smetric_policy, P, P,
                                                     P, P, P, P, I64, P]),
            "smetric_index_commit_batch": (C.c_int, [P, P, I32, P, P, P, I32, P, P]),
            "smetric_index_set_lru": (C.c_int, [P, I64, I64]),
            "smetric_route_commit_batch": (C.c_int, [P, P, I64, P, I32, P, smetric_weights, P, P, P, P, P, I64,
                                                     I32, P]),
            "smetric_index_lru_sizes": (C.c_int, [P, P, P]),
            "smetric_link_sessions": (C.c_int, [P, P, I64, P, I32, P, P, P, P, P]),
            "smetric_reuse_workspace_bytes": (I64, [I64]),
            "smetric_imbalance_workspace_bytes": (I64, [I32, I32]),
            "smetric_window_imbalance": (C.c_int, [P, P, P, P, I32, I64, I32, P, I64, P, P, P, P]),
            "smetric_reuse_breakdown": (C.c_int, [P, P, I64, P, I32, P, P, P, I64, P, P, P, P, P]),
            "smetric_route_batch_sequential": (C.c_int, [P, P, I64, P, I32, P, smetric_weights, P, P, P, P, P,
                                                         I64, P, P]),
            "smetric_route_batch_baseline": (C.c_int, [P, P, I64, P, I32, I32, P, P, I64, I64, P, P, P, P, P,
                                                       I64, P]),
            "smetric_route_batch_policy_coloc": (C.c_int, [P, P, I64, P, I32, P, P, P, P, P, smetric_policy,
                                                           P, P, P, P, P, P, I64, P]),
            "smetric_block_hashes": (C.c_int, [P, P, I64, P, I32, P, P, I64, P]),
            "smetric_block_hashes_noalloc": (C.c_int, [P, I64, P, I32, I32, I32, C.c_uint64, P, P, I64,
                                                      P, P]),
            "smetric_route_batch_host": (C.c_int, [P, P, I64, P, I32, P, smetric_weights, P, P, P,
                                                   P, P]),
            "smetric_status": (C.c_int, [P, P]),
            "smetric_strerror": (C.c_char_p, [C.c_int]),
            "smetric_profile_enable": (C.c_int, [P, I32]),
            "smetric_profile_read": (C.c_int, [P, I32, P, P]),
            "smetric_profile_kernel_name": (C.c_char_p, [I32]),
            "smetric_launch_count": (I64, [P]),
            "smetric_kv_create": (C.c_int, [C.POINTER(smetric_kv_config), C.POINTER(P)]),
            "smetric_kv_destroy": (C.c_int, [P]),
            "smetric_kv_plan": (C.c_int, [P, P, I32, I64, P, P, I32, I64, I32, P]),
            "smetric_kv_plan_up_to": (C.c_int, [P, P, I32, I64, P, P, I32, I64, I32, I64, P]),
            "smetric_kv_append": (C.c_int, [P, smetric_kv_cache, smetric_heads, smetric_heads, smetric_heads,
                                            smetric_heads, smetric_kv_transform, P]),
            "smetric_qk_norm_rope": (C.c_int, [P, smetric_heads, smetric_heads, P, I64, smetric_kv_transform,
                                               smetric_heads, smetric_heads, P]),
            "smetric_paged_attention": (C.c_int, [P, smetric_kv_cache, smetric_heads, C.c_float, smetric_heads, P,
                                                  P]),
            "smetric_kvq_append": (C.c_int, [P, smetric_kvq_cache, smetric_kvq_cache, smetric_heads, smetric_heads,
                                             smetric_heads, smetric_heads, smetric_kv_transform, P]),
            "smetric_kvq_read": (C.c_int, [P, smetric_kvq_cache, smetric_kvq_cache, P, I32, I64, P, P, I32, I64,
                                           smetric_heads, smetric_heads, P]),
            "smetric_kvq_attention": (C.c_int, [P, smetric_kvq_cache, smetric_kvq_cache, smetric_heads, C.c_float,
                                                smetric_heads, P, P]),
            "smetric_kv_status": (C.c_int, [P, P]),
            "smetric_kv_launch_count": (I64, [P]),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


# ---------------------------------------------------------------------------
# marshalling helpers
# ---------------------------------------------------------------------------

def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        if not x.is_contiguous():
            raise ValueError("arrays must be contiguous")
        return x.data_ptr() if x.numel() > 0 else None
    if hasattr(x, "ctypes"):  # numpy array (host memory)
        return x.ctypes.data if x.size > 0 else None
    raise TypeError(f"cannot pass {type(x)} as a pointer")


def _stream(s) -> Optional[int]:
    if s is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(rc: int, where: str):
    if rc != SMETRIC_OK:
        raise SmetricError(rc, where)


def _weights(w) -> smetric_weights:
    if isinstance(w, smetric_weights):
        return w
    a, b, c = w
    return smetric_weights(int(a), int(b), int(c))


# ---------------------------------------------------------------------------
# C ABI, one function per entry point
# ---------------------------------------------------------------------------

def smetric_index_create(cfg: smetric_index_config) -> int:
    h = C.c_void_p()
    _check(lib().smetric_index_create(C.byref(cfg), C.byref(h)), "smetric_index_create")
    return h.value


def smetric_index_destroy(idx: int) -> None:
    _check(lib().smetric_index_destroy(idx), "smetric_index_destroy")


def smetric_index_clear(idx: int, stream=None) -> None:
    _check(lib().smetric_index_clear(idx, _stream(stream)), "smetric_index_clear")


def smetric_index_insert(idx: int, d_keys, d_tiers, n: int, stream=None) -> None:
    _check(lib().smetric_index_insert(idx, _ptr(d_keys), _ptr(d_tiers), n, _stream(stream)),
           "smetric_index_insert")


def smetric_index_evict(idx: int, d_keys, d_tiers, n: int, stream=None) -> None:
    _check(lib().smetric_index_evict(idx, _ptr(d_keys), _ptr(d_tiers), n, _stream(stream)),
           "smetric_index_evict")


def smetric_index_lookup(idx: int, d_keys, n: int, d_masks, stream=None) -> None:
    _check(lib().smetric_index_lookup(idx, _ptr(d_keys), n, _ptr(d_masks), _stream(stream)),
           "smetric_index_lookup")


def smetric_index_mask_words(idx: int) -> int:
    return int(lib().smetric_index_mask_words(idx))


def smetric_route_batch(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int, d_load,
                        w, d_instance, d_local_hit, d_global_hit, d_session_key,
                        d_block_hashes=None, hashes_cap: int = 0, stream=None) -> None:
    _check(lib().smetric_route_batch(idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests,
                                     _ptr(d_load), _weights(w), _ptr(d_instance), _ptr(d_local_hit),
                                     _ptr(d_global_hit), _ptr(d_session_key), _ptr(d_block_hashes),
                                     hashes_cap, _stream(stream)), "smetric_route_batch")


def smetric_route_commit_batch(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int, d_load, w,
                               d_instance, d_local_hit, d_global_hit, d_session_key, d_block_hashes,
                               hashes_cap: int, flags: int = 0, stream=None) -> None:
    _check(lib().smetric_route_commit_batch(idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests,
                                            _ptr(d_load), _weights(w), _ptr(d_instance), _ptr(d_local_hit),
                                            _ptr(d_global_hit), _ptr(d_session_key), _ptr(d_block_hashes),
                                            hashes_cap, flags, _stream(stream)), "smetric_route_commit_batch")


def smetric_route_batches(idx: int, d_tokens, n_tokens, d_offsets, n_requests, d_load, w, d_instance,
                          d_local_hit, d_global_hit, d_session_key, stream=None) -> None:
    """Several batches in one call; every argument but idx, w and stream is a
    sequence with one entry per batch (device arrays, or counts)."""
    nb = len(n_requests)
    if not all(len(x) == nb for x in (d_tokens, n_tokens, d_offsets, d_load, d_instance, d_local_hit,
                                      d_global_hit, d_session_key)):
        raise ValueError("every per-batch sequence needs one entry per batch")
    ptrs = lambda xs: (C.c_void_p * max(nb, 1))(*[_ptr(x) for x in xs])
    _check(lib().smetric_route_batches(idx, nb, ptrs(d_tokens), (C.c_int64 * max(nb, 1))(*n_tokens),
                                       ptrs(d_offsets), (C.c_int32 * max(nb, 1))(*n_requests), ptrs(d_load),
                                       _weights(w), ptrs(d_instance), ptrs(d_local_hit), ptrs(d_global_hit),
                                       ptrs(d_session_key), _stream(stream)), "smetric_route_batches")


def _policy(p) -> smetric_policy:
    if isinstance(p, smetric_policy):
        return p
    d = dict(p)
    return smetric_policy(int(d["c_lin"]), int(d["c_att"]), int(d["ttft_d0"]), int(d["ttft_d1"]),
                          int(d["hit_num"]), int(d["hit_den"]), int(d.get("rr_base", 0)), 0)


def smetric_route_batch_policy(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int,
                               d_queued, d_turn, d_est_hit, policy, d_instance, d_local_hit,
                               d_global_hit, d_stick, d_session_key, d_block_hashes=None,
                               hashes_cap: int = 0, stream=None) -> None:
    _check(lib().smetric_route_batch_policy(
        idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests, _ptr(d_queued), _ptr(d_turn),
        _ptr(d_est_hit), _policy(policy), _ptr(d_instance), _ptr(d_local_hit), _ptr(d_global_hit),
        _ptr(d_stick), _ptr(d_session_key), _ptr(d_block_hashes), hashes_cap, _stream(stream)),
        "smetric_route_batch_policy")


def smetric_route_batch_policy_coloc(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int,
                                     d_queued, d_tpot_budget, d_num_requests, d_turn, d_est_hit, policy,
                                     d_instance, d_local_hit, d_global_hit, d_stick, d_session_key,
                                     d_block_hashes=None, hashes_cap: int = 0, stream=None) -> None:
    _check(lib().smetric_route_batch_policy_coloc(
        idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests, _ptr(d_queued), _ptr(d_tpot_budget),
        _ptr(d_num_requests), _ptr(d_turn), _ptr(d_est_hit), _policy(policy), _ptr(d_instance),
        _ptr(d_local_hit), _ptr(d_global_hit), _ptr(d_stick), _ptr(d_session_key), _ptr(d_block_hashes),
        hashes_cap, _stream(stream)), "smetric_route_batch_policy_coloc")


def smetric_route_batch_baseline(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int, scorer: int,
                                 d_queued, d_batch, lam_num: int, lam_den: int, d_instance, d_local_hit,
                                 d_global_hit, d_session_key, d_block_hashes=None, hashes_cap: int = 0,
                                 stream=None) -> None:
    _check(lib().smetric_route_batch_baseline(
        idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests, scorer, _ptr(d_queued), _ptr(d_batch),
        lam_num, lam_den, _ptr(d_instance), _ptr(d_local_hit), _ptr(d_global_hit), _ptr(d_session_key),
        _ptr(d_block_hashes), hashes_cap, _stream(stream)), "smetric_route_batch_baseline")


def smetric_route_batch_sequential(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int, d_load, w,
                                   d_instance, d_local_hit, d_global_hit, d_session_key, d_block_hashes=None,
                                   hashes_cap: int = 0, d_load_after=None, stream=None) -> None:
    _check(lib().smetric_route_batch_sequential(
        idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests, _ptr(d_load), _weights(w), _ptr(d_instance),
        _ptr(d_local_hit), _ptr(d_global_hit), _ptr(d_session_key), _ptr(d_block_hashes), hashes_cap,
        _ptr(d_load_after), _stream(stream)), "smetric_route_batch_sequential")


def smetric_reuse_workspace_bytes(n_blocks: int) -> int:
    return int(lib().smetric_reuse_workspace_bytes(n_blocks))


def smetric_reuse_breakdown(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int, d_sessions,
                            d_sys_blocks, d_workspace, workspace_bytes: int, d_hit, d_sys, d_intra, d_inter,
                            stream=None) -> None:
    _check(lib().smetric_reuse_breakdown(idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests,
                                         _ptr(d_sessions), _ptr(d_sys_blocks), _ptr(d_workspace), workspace_bytes,
                                         _ptr(d_hit), _ptr(d_sys), _ptr(d_intra), _ptr(d_inter), _stream(stream)),
           "smetric_reuse_breakdown")


def smetric_imbalance_workspace_bytes(n_windows: int, num_instances: int) -> int:
    return int(lib().smetric_imbalance_workspace_bytes(n_windows, num_instances))


def smetric_window_imbalance(idx: int, d_instance, d_start, d_end, n_requests: int, window: int, n_windows: int,
                             d_workspace, workspace_bytes: int, d_max, d_argmax, d_sum, stream=None) -> None:
    _check(lib().smetric_window_imbalance(idx, _ptr(d_instance), _ptr(d_start), _ptr(d_end), n_requests, window,
                                          n_windows, _ptr(d_workspace), workspace_bytes, _ptr(d_max),
                                          _ptr(d_argmax), _ptr(d_sum), _stream(stream)),
           "smetric_window_imbalance")


def smetric_link_sessions(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int, d_users, d_turns,
                          d_parent, d_session, stream=None) -> None:
    _check(lib().smetric_link_sessions(idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests, _ptr(d_users),
                                       _ptr(d_turns), _ptr(d_parent), _ptr(d_session), _stream(stream)),
           "smetric_link_sessions")


def smetric_index_commit_batch(idx: int, d_offsets, n_requests: int, d_instance, d_local_hit,
                               d_block_hashes, flags: int = 0, d_load=None, stream=None) -> None:
    _check(lib().smetric_index_commit_batch(idx, _ptr(d_offsets), n_requests, _ptr(d_instance),
                                            _ptr(d_local_hit), _ptr(d_block_hashes), flags, _ptr(d_load),
                                            _stream(stream)), "smetric_index_commit_batch")


def smetric_index_set_lru(idx: int, local_cap: int, global_cap: int) -> None:
    _check(lib().smetric_index_set_lru(idx, local_cap, global_cap), "smetric_index_set_lru")


def smetric_index_lru_sizes(idx: int, d_sizes, stream=None) -> None:
    _check(lib().smetric_index_lru_sizes(idx, _ptr(d_sizes), _stream(stream)), "smetric_index_lru_sizes")


def smetric_block_hashes(idx: int, d_tokens, n_tokens: int, d_offsets, n_requests: int,
                         d_session_key, d_block_hashes, hashes_cap: int, stream=None) -> None:
    _check(lib().smetric_block_hashes(idx, _ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests,
                                      _ptr(d_session_key), _ptr(d_block_hashes), hashes_cap,
                                      _stream(stream)), "smetric_block_hashes")


def smetric_block_hashes_noalloc(d_tokens, n_tokens: int, d_offsets, n_requests: int,
                                 block_size: int, session_blocks: int, hash_seed: int,
                                 d_session_key, d_block_hashes, hashes_cap: int, d_status,
                                 stream=None) -> int:
    """Returns the call's host-side status code (SMETRIC_ERR_TOO_LARGE for a
    batch beyond the fixed scratch); device-detected errors land in d_status."""
    return int(lib().smetric_block_hashes_noalloc(_ptr(d_tokens), n_tokens, _ptr(d_offsets), n_requests,
                                                  block_size, session_blocks, hash_seed,
                                                  _ptr(d_session_key), _ptr(d_block_hashes), hashes_cap,
                                                  _ptr(d_status), _stream(stream)))


def smetric_route_batch_host(idx: int, h_tokens, n_tokens: int, h_offsets, n_requests: int, h_load,
                             w, h_instance, h_local_hit, h_global_hit, h_session_key,
                             stream=None) -> int:
    """Returns the call's status (device-latched errors included)."""
    return int(lib().smetric_route_batch_host(idx, _ptr(h_tokens), n_tokens, _ptr(h_offsets),
                                              n_requests, _ptr(h_load), _weights(w),
                                              _ptr(h_instance), _ptr(h_local_hit),
                                              _ptr(h_global_hit), _ptr(h_session_key),
                                              _stream(stream)))


def smetric_status(idx: int, stream=None) -> int:
    return int(lib().smetric_status(idx, _stream(stream)))


def smetric_strerror(code: int) -> str:
    return lib().smetric_strerror(code).decode()


def smetric_profile_enable(idx: int, on: bool) -> None:
    _check(lib().smetric_profile_enable(idx, 1 if on else 0), "smetric_profile_enable")


def smetric_profile_read(idx: int):
    """{kernel name: (milliseconds, launches)} since the previous read."""
    ms = (C.c_double * 8)()
    ln = (C.c_int64 * 8)()
    k = lib().smetric_profile_read(idx, 8, ms, ln)
    if k < 0:
        raise SmetricError(k, "smetric_profile_read")
    return {smetric_profile_kernel_name(i): (ms[i], ln[i]) for i in range(k)}


def smetric_profile_kernel_name(k: int) -> str:
    return lib().smetric_profile_kernel_name(k).decode()


def smetric_launch_count(idx: int) -> int:
    return int(lib().smetric_launch_count(idx))


def smetric_kv_create(cfg: smetric_kv_config) -> int:
    h = C.c_void_p()
    _check(lib().smetric_kv_create(C.byref(cfg), C.byref(h)), "smetric_kv_create")
    return h.value


def smetric_kv_destroy(kv: int) -> None:
    _check(lib().smetric_kv_destroy(kv), "smetric_kv_destroy")


def smetric_kv_plan(kv: int, d_offsets, n_requests: int, n_tokens: int, d_kv_lens, d_pages, max_pages: int,
                    pages_stride: int, window: int = 0, stream=None) -> None:
    _check(lib().smetric_kv_plan(kv, _ptr(d_offsets), n_requests, n_tokens, _ptr(d_kv_lens), _ptr(d_pages), max_pages,
                                 pages_stride, window, _stream(stream)), "smetric_kv_plan")


def smetric_kv_plan_up_to(kv: int, d_offsets, n_requests: int, n_tokens: int, d_kv_lens, d_pages, max_pages: int,
                          pages_stride: int, window: int, max_new: int, stream=None) -> None:
    _check(lib().smetric_kv_plan_up_to(kv, _ptr(d_offsets), n_requests, n_tokens, _ptr(d_kv_lens), _ptr(d_pages), max_pages,
                                       pages_stride, window, max_new, _stream(stream)), "smetric_kv_plan_up_to")


def smetric_kv_append(kv: int, cache: smetric_kv_cache, k: smetric_heads, v: smetric_heads, q: smetric_heads,
                      q_out: smetric_heads, transform: smetric_kv_transform, stream=None) -> None:
    _check(lib().smetric_kv_append(kv, cache, k, v, q, q_out, transform, _stream(stream)), "smetric_kv_append")


def smetric_qk_norm_rope(kv: int, q: smetric_heads, k: smetric_heads, d_positions, n_tokens: int,
                         transform: smetric_kv_transform, q_out: smetric_heads, k_out: smetric_heads,
                         stream=None) -> None:
    _check(lib().smetric_qk_norm_rope(kv, q, k, _ptr(d_positions), n_tokens, transform, q_out, k_out,
                                      _stream(stream)), "smetric_qk_norm_rope")


def smetric_paged_attention(kv: int, cache: smetric_kv_cache, q: smetric_heads, scale: float, out: smetric_heads,
                            d_lse=None, stream=None) -> None:
    _check(lib().smetric_paged_attention(kv, cache, q, scale, out, _ptr(d_lse), _stream(stream)),
           "smetric_paged_attention")


def smetric_kvq_append(kv: int, k_cache: smetric_kvq_cache, v_cache: smetric_kvq_cache, k: smetric_heads, v: smetric_heads,
                       q: smetric_heads, q_out: smetric_heads, transform: smetric_kv_transform, stream=None) -> None:
    _check(lib().smetric_kvq_append(kv, k_cache, v_cache, k, v, q, q_out, transform, _stream(stream)), "smetric_kvq_append")


def smetric_kvq_read(kv: int, k_cache: smetric_kvq_cache, v_cache: smetric_kvq_cache, d_offsets, n_requests: int, n_rows: int,
                     d_first, d_pages, max_pages: int, pages_stride: int, k: smetric_heads, v: smetric_heads,
                     stream=None) -> None:
    _check(lib().smetric_kvq_read(kv, k_cache, v_cache, _ptr(d_offsets), n_requests, n_rows, _ptr(d_first), _ptr(d_pages),
                                  max_pages, pages_stride, k, v, _stream(stream)), "smetric_kvq_read")


def smetric_kvq_attention(kv: int, k_cache: smetric_kvq_cache, v_cache: smetric_kvq_cache, q: smetric_heads, scale: float,
                          out: smetric_heads, d_lse=None, stream=None) -> None:
    _check(lib().smetric_kvq_attention(kv, k_cache, v_cache, q, scale, out, _ptr(d_lse), _stream(stream)),
           "smetric_kvq_attention")


def smetric_kv_status(kv: int, stream=None) -> int:
    return int(lib().smetric_kv_status(kv, _stream(stream)))


def smetric_kv_launch_count(kv: int) -> int:
    return int(lib().smetric_kv_launch_count(kv))


# ---------------------------------------------------------------------------
# convenience wrappers
# ---------------------------------------------------------------------------

class SMetricIndex:
    """One two-tier index on the current CUDA device, with torch outputs."""

    def __init__(self, num_instances: int, block_size: int, session_blocks: int,
                 capacity_slots: int, max_batch_requests: int, max_batch_tokens: int,
                 hash_seed: int = 0, host_staging: bool = False, pipeline: bool = False):
        self.cfg = smetric_index_config(num_instances, block_size, session_blocks,
                                        (SMETRIC_FLAG_HOST_STAGING if host_staging else 0)
                                        | (SMETRIC_FLAG_PIPELINE if pipeline else 0),
                                        capacity_slots, hash_seed & 0xFFFFFFFFFFFFFFFF,
                                        max_batch_requests, max_batch_tokens)
        self.handle = smetric_index_create(self.cfg)
        self.N, self.B, self.S = num_instances, block_size, session_blocks
        self.W = smetric_index_mask_words(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            smetric_index_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _tiers(self, keys, tiers):
        import torch
        if isinstance(tiers, int):
            tiers = torch.full(keys.shape, tiers, dtype=torch.int32, device=keys.device)
        return tiers

    def insert(self, keys, tiers, stream=None):
        tiers = self._tiers(keys, tiers)
        smetric_index_insert(self.handle, keys, tiers, keys.numel(), stream)

    def evict(self, keys, tiers, stream=None):
        tiers = self._tiers(keys, tiers)
        smetric_index_evict(self.handle, keys, tiers, keys.numel(), stream)

    def clear(self, stream=None):
        smetric_index_clear(self.handle, stream)

    def lookup(self, keys, stream=None):
        import torch
        out = torch.empty((keys.numel(), self.W), dtype=torch.uint64, device=keys.device)
        smetric_index_lookup(self.handle, keys, keys.numel(), out, stream)
        return out

    def route_batches(self, batches, weights=(1, 4, 2), out=None, stream=None):
        """Routes a list of (tokens, offsets, load) device batches in one call;
        returns one dict(instance, local_hit, global_hit, session_key) per
        batch (or fills `out`, a list of such dicts)."""
        import torch
        if out is None:
            out = []
            for tokens, offsets, _ in batches:
                n, dev = offsets.numel() - 1, offsets.device
                out.append(dict(instance=torch.empty(n, dtype=torch.int32, device=dev),
                                local_hit=torch.empty(n, dtype=torch.int32, device=dev),
                                global_hit=torch.empty(n, dtype=torch.int32, device=dev),
                                session_key=torch.empty(n, dtype=torch.uint64, device=dev)))
        smetric_route_batches(self.handle, [b[0] for b in batches], [b[0].numel() for b in batches],
                              [b[1] for b in batches], [b[1].numel() - 1 for b in batches],
                              [b[2] for b in batches], weights, [o["instance"] for o in out],
                              [o["local_hit"] for o in out], [o["global_hit"] for o in out],
                              [o["session_key"] for o in out], stream)
        return out

    def route_batch(self, tokens, offsets, load, weights=(1, 4, 2), want_hashes=False,
                    out=None, stream=None):
        """Returns dict(instance, local_hit, global_hit, session_key[, block_hashes])."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        if out is None:
            out = dict(instance=torch.empty(n, dtype=torch.int32, device=dev),
                       local_hit=torch.empty(n, dtype=torch.int32, device=dev),
                       global_hit=torch.empty(n, dtype=torch.int32, device=dev),
                       session_key=torch.empty(n, dtype=torch.uint64, device=dev))
            if want_hashes:
                out["block_hashes"] = torch.empty(max(tokens.numel() // self.B, 1),
                                                  dtype=torch.uint64, device=dev)
        hb = out.get("block_hashes")
        smetric_route_batch(self.handle, tokens, tokens.numel(), offsets, n, load, weights,
                            out["instance"], out["local_hit"], out["global_hit"],
                            out["session_key"], hb, hb.numel() if hb is not None else 0, stream)
        return out

    def route_commit_batch(self, tokens, offsets, load, weights=(1, 4, 2), also_global=False, stream=None):
        """route_batch then commit_batch on the device in one call; `load` is
        read by the route and drained in place. Returns route_batch's dict
        with block_hashes."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        out = dict(instance=torch.empty(n, dtype=torch.int32, device=dev),
                   local_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   global_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   session_key=torch.empty(n, dtype=torch.uint64, device=dev),
                   block_hashes=torch.empty(max(tokens.numel() // self.B, 1), dtype=torch.uint64, device=dev))
        hb = out["block_hashes"]
        smetric_route_commit_batch(self.handle, tokens, tokens.numel(), offsets, n, load, weights, out["instance"],
                                   out["local_hit"], out["global_hit"], out["session_key"], hb, hb.numel(),
                                   SMETRIC_COMMIT_GLOBAL if also_global else 0, stream)
        return out

    def route_batch_policy(self, tokens, offsets, queued, turn, est_hit, policy, want_hashes=False,
                           out=None, stream=None):
        """The session-centric policy (Figure 10). `policy` is a dict with c_lin,
        c_att, ttft_d0, ttft_d1, hit_num, hit_den and optionally rr_base.
        Returns dict(instance, local_hit, global_hit, stick, session_key[, block_hashes])."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        if out is None:
            out = dict(instance=torch.empty(n, dtype=torch.int32, device=dev),
                       local_hit=torch.empty(n, dtype=torch.int32, device=dev),
                       global_hit=torch.empty(n, dtype=torch.int32, device=dev),
                       stick=torch.empty(n, dtype=torch.int32, device=dev),
                       session_key=torch.empty(n, dtype=torch.uint64, device=dev))
            if want_hashes:
                out["block_hashes"] = torch.empty(max(tokens.numel() // self.B, 1),
                                                  dtype=torch.uint64, device=dev)
        hb = out.get("block_hashes")
        smetric_route_batch_policy(self.handle, tokens, tokens.numel(), offsets, n, queued, turn, est_hit,
                                   policy, out["instance"], out["local_hit"], out["global_hit"],
                                   out["stick"], out["session_key"], hb,
                                   hb.numel() if hb is not None else 0, stream)
        return out

    def route_batch_policy_coloc(self, tokens, offsets, queued, tpot_budget, num_requests, turn, est_hit,
                                 policy, want_hashes=False, stream=None):
        """The session-centric policy under PD colocation (Appendix B).
        Returns dict(instance, local_hit, global_hit, stick, session_key[, block_hashes])."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        out = dict(instance=torch.empty(n, dtype=torch.int32, device=dev),
                   local_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   global_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   stick=torch.empty(n, dtype=torch.int32, device=dev),
                   session_key=torch.empty(n, dtype=torch.uint64, device=dev))
        if want_hashes:
            out["block_hashes"] = torch.empty(max(tokens.numel() // self.B, 1), dtype=torch.uint64, device=dev)
        hb = out.get("block_hashes")
        smetric_route_batch_policy_coloc(self.handle, tokens, tokens.numel(), offsets, n, queued, tpot_budget,
                                         num_requests, turn, est_hit, policy, out["instance"], out["local_hit"],
                                         out["global_hit"], out["stick"], out["session_key"], hb,
                                         hb.numel() if hb is not None else 0, stream)
        return out

    def route_batch_baseline(self, tokens, offsets, scorer, queued, batch, lam=(1, 2), stream=None):
        """A baseline scorer of Section 5.1 (SMETRIC_SCORER_BAILIAN or _LMETRIC).
        Returns dict(instance, local_hit, global_hit, session_key)."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        out = dict(instance=torch.empty(n, dtype=torch.int32, device=dev),
                   local_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   global_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   session_key=torch.empty(n, dtype=torch.uint64, device=dev))
        smetric_route_batch_baseline(self.handle, tokens, tokens.numel(), offsets, n, scorer, queued, batch,
                                     lam[0], lam[1], out["instance"], out["local_hit"], out["global_hit"],
                                     out["session_key"], None, 0, stream)
        return out

    def route_batch_sequential(self, tokens, offsets, load, weights=(1, 4, 2), stream=None):
        """The argmin cost with loads updated request by request. Returns
        dict(instance, local_hit, global_hit, session_key, load_after)."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        out = dict(instance=torch.empty(n, dtype=torch.int32, device=dev),
                   local_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   global_hit=torch.empty(n, dtype=torch.int32, device=dev),
                   session_key=torch.empty(n, dtype=torch.uint64, device=dev),
                   load_after=torch.empty(self.N, dtype=torch.int64, device=dev))
        smetric_route_batch_sequential(self.handle, tokens, tokens.numel(), offsets, n, load, weights,
                                       out["instance"], out["local_hit"], out["global_hit"], out["session_key"],
                                       None, 0, out["load_after"], stream)
        return out

    def reuse_breakdown(self, tokens, offsets, sessions, sys_blocks, workspace=None, stream=None):
        """KV$ reuse against an unbounded store of the earlier requests:
        dict(hit, sys, intra, inter), int32 blocks per request."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        need = smetric_reuse_workspace_bytes(tokens.numel() // self.B)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        out = {k: torch.empty(n, dtype=torch.int32, device=dev) for k in ("hit", "sys", "intra", "inter")}
        smetric_reuse_breakdown(self.handle, tokens, tokens.numel(), offsets, n, sessions, sys_blocks, workspace,
                                workspace.numel(), out["hit"], out["sys"], out["intra"], out["inter"], stream)
        return out

    def window_imbalance(self, instance, start, end, window: int, n_windows: int, workspace=None, stream=None):
        """Per window: dict(max, argmax, sum) of the instances' running-request
        ticks; the imbalance is N * max / sum."""
        import torch
        dev = start.device
        if workspace is None:
            workspace = torch.empty(max(1, smetric_imbalance_workspace_bytes(n_windows, self.N) // 8),
                                    dtype=torch.int64, device=dev)
        out = dict(max=torch.empty(n_windows, dtype=torch.int64, device=dev),
                   argmax=torch.empty(n_windows, dtype=torch.int32, device=dev),
                   sum=torch.empty(n_windows, dtype=torch.int64, device=dev))
        smetric_window_imbalance(self.handle, instance, start, end, instance.numel(), window, n_windows, workspace,
                                 workspace.numel() * workspace.element_size(), out["max"], out["argmax"],
                                 out["sum"], stream)
        return out

    def link_sessions(self, tokens, offsets, users, turns, stream=None):
        """Session reconstruction (Appendix A): returns (parent, session), int32 per request."""
        import torch
        n = offsets.numel() - 1
        parent = torch.empty(n, dtype=torch.int32, device=offsets.device)
        session = torch.empty(n, dtype=torch.int32, device=offsets.device)
        smetric_link_sessions(self.handle, tokens, tokens.numel(), offsets, n, users, turns, parent, session,
                              stream)
        return parent, session

    def commit_batch(self, offsets, out, also_global=False, load=None, stream=None):
        """Add the routed batch's blocks (`out` from route_batch(..., want_hashes=True)
        or route_batch_policy) to its chosen instances' local tiers (and the
        global tier); with `load`, drain it in place."""
        smetric_index_commit_batch(self.handle, offsets, offsets.numel() - 1, out["instance"],
                                   out["local_hit"], out["block_hashes"],
                                   SMETRIC_COMMIT_GLOBAL if also_global else 0, load, stream)

    def set_lru(self, local_cap=0, global_cap=0):
        """Caps the local tiers at `local_cap` blocks each and the global tier
        at `global_cap` (0: uncapped); commit_batch then evicts each capped
        tier's least recently used blocks on the device."""
        smetric_index_set_lru(self.handle, int(local_cap), int(global_cap))

    def lru_sizes(self, stream=None):
        """Blocks the device LRU tracks per tier (int64 [N+1], global last)."""
        import torch
        out = torch.empty(self.N + 1, dtype=torch.int64, device="cuda")
        smetric_index_lru_sizes(self.handle, out, stream)
        return out

    def block_hashes(self, tokens, offsets, stream=None):
        """Returns (block_hashes, session_key) as device tensors."""
        import torch
        n = offsets.numel() - 1
        dev = offsets.device
        hb = torch.empty(max(tokens.numel() // self.B, 1), dtype=torch.uint64, device=dev)
        sk = torch.empty(max(n, 1), dtype=torch.uint64, device=dev)
        smetric_block_hashes(self.handle, tokens, tokens.numel(), offsets, n, sk, hb, hb.numel(),
                             stream)
        return hb, sk[:n]

    def status(self, stream=None) -> int:
        return smetric_status(self.handle, stream)

    def check(self, stream=None):
        rc = self.status(stream)
        if rc != SMETRIC_OK:
            raise SmetricError(rc, "device")


_NO_HEADS = smetric_heads()


class SMetricKV:
    """The paged KV$ operators for one layout of heads and pages, with torch
    tensors. Caches are [num_pages, page_size, num_kv_heads, head_dim] views
    (any strides but the last), heads [tokens, heads, head_dim] views.

        kv = SMetricKV(head_dim=128, num_q_heads=32, num_kv_heads=4, page_size=32, num_pages=4096,
                       max_batch_requests=64, max_batch_tokens=8192)
        kv.plan(offsets_i64, kv_lens_i32, pages_i32, n_tokens)       # once a step
        kv.append(k_cache, v_cache, k, v, q=q, q_out=q, cos_sin=table, q_norm=wq, k_norm=wk)
        out = kv.paged_attention(q, k_cache, v_cache)
        kv.check()

    Tensors are on the device that was current when the object was made. A call
    on another stream than torch's current one (stream=) allocates its new
    outputs there; the caller orders the two streams, as for its inputs.
    """

    _flags = 0
    _append_call, _attention_call = "smetric_kv_append", "smetric_paged_attention"

    def __init__(self, head_dim: int, num_q_heads: int, num_kv_heads: int, page_size: int, num_pages: int,
                 max_batch_requests: int, max_batch_tokens: int, dtype=None):
        import torch
        self.dtype = torch.bfloat16 if dtype is None else dtype
        code = {torch.bfloat16: SMETRIC_BF16, torch.float16: SMETRIC_F16}.get(self.dtype)
        if code is None:
            raise ValueError("dtype must be torch.bfloat16 or torch.float16")
        self.cfg = smetric_kv_config(head_dim, num_q_heads, num_kv_heads, page_size, code, self._flags, num_pages,
                                     max_batch_requests, max_batch_tokens)
        self.handle = smetric_kv_create(self.cfg)
        self._n_tokens = None
        # the plan's tensors; torch's current stream when they were given; reads of them on others, as events
        # after the last one; and the tensors of plans before, with such events
        self._kept, self._home, self._reads, self._dropped = None, None, {}, []
        # (what the calls use each time: a step's few tokens are bound by the host)
        self._lib, self._raw_stream, self._device = lib(), torch._C._cuda_getCurrentRawStream, torch.cuda.current_device()
        self._dim, self._f32, self._i32 = head_dim, torch.float32, torch.int32
        self._empty, self._like = torch.empty, torch.empty_like
        self._others = {}  # torch's objects for streams given by a call, by their raw ones
        self._cache_shape = (num_pages, page_size, num_kv_heads, head_dim)

    def close(self):
        if getattr(self, "handle", None):
            smetric_kv_destroy(self.handle)  # (waits for the device)
            self.handle = None
            self._kept, self._reads, self._dropped = None, {}, []

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _heads(self, x, heads: int, n_tokens: int, name: str) -> smetric_heads:
        if x is None:
            return _NO_HEADS
        if x.dtype != self.dtype or x.shape != (n_tokens, heads, self._dim) or x.get_device() != self._device:
            raise ValueError(f"{name} must be {self.dtype} [{n_tokens}, {heads}, {self._dim}] on cuda:{self._device}")
        token, head, one = x.stride()
        if one != 1 and x.numel():
            raise ValueError(f"{name}: the elements of a head must be contiguous")
        # (the stride of a dimension of one is arbitrary)
        return smetric_heads(x.data_ptr(), token if n_tokens > 1 else 0, head if heads > 1 else 0)

    def _caches(self, k_cache, v_cache):
        return (self._cache(k_cache, v_cache),)

    def _cache(self, k_cache, v_cache) -> smetric_kv_cache:
        shape = self._cache_shape
        here = self._device
        if (k_cache.dtype != self.dtype or v_cache.dtype != self.dtype or k_cache.shape != shape or v_cache.shape != shape or
                k_cache.get_device() != here or v_cache.get_device() != here):
            raise ValueError(f"caches must be {self.dtype} {list(shape)} on cuda:{here}")
        strides = k_cache.stride()
        if v_cache.stride() != strides or strides[3] != 1:
            raise ValueError("caches must have equal strides and contiguous heads")
        return smetric_kv_cache(k_cache.data_ptr(), v_cache.data_ptr(), strides[0] if shape[0] > 1 else 0, strides[1],
                                strides[2] if shape[2] > 1 else 0)

    def _stream(self, stream):
        """A call's stream: (raw, None), or (raw, torch's object for it) where it is not torch's current one."""
        now = self._raw_stream(self._device)
        if stream is None:
            return now, None
        raw = _stream(stream)
        if raw == 1:  # (the legacy default stream by its other name)
            raw = 0
        if raw == now:
            return raw, None
        return raw, self._object(raw)

    def _object(self, raw: int):
        s = self._others.get(raw)
        if s is None:
            import torch
            s = self._others[raw] = torch.cuda.ExternalStream(raw, device=self._device)
        return s

    def _read(self, raw: int, other):
        """Notes that a call on a stream reads the plan's tensors. Where it is not
        the one that they were given on, they are to outlive the call."""
        if raw == self._home:
            return
        import torch
        now = torch.cuda.current_stream(self._device)
        if other is not None:
            torch.cuda.set_stream(other)
        try:
            if not torch.cuda.is_current_stream_capturing():
                done = self._reads.get(raw)
                if done is None:
                    done = self._reads[raw] = torch.cuda.Event()
                done.record(self._object(raw))
        finally:
            if other is not None:
                torch.cuda.set_stream(now)

    def _keep(self, tensors):
        """Holds a plan's tensors, and those of plans before it that are still read on another stream."""
        import torch
        if self._reads:
            self._dropped.append((self._kept, list(self._reads.values())))
            self._reads = {}
        if self._dropped and not torch.cuda.is_current_stream_capturing():
            self._dropped = [x for x in self._dropped if not all(e.query() for e in x[1])]
        self._kept, self._home = tensors, self._raw_stream(self._device)

    def _new(self, other, make, *args, **kw):
        """A new tensor for a call on the stream `other` to fill (None: torch's
        current one). Its memory is that stream's, as what was done with it
        before may still wait on the current one; and goes back to it only when
        the current stream is done with it too."""
        import torch
        if other is None or torch.cuda.current_device() != self._device:  # (a call that is refused)
            return make(*args, **kw)
        now = torch.cuda.current_stream(self._device)
        torch.cuda.set_stream(other)  # (the context manager costs the host 5 us more)
        try:
            x = make(*args, **kw)
        finally:
            torch.cuda.set_stream(now)
        x.record_stream(now)
        return x

    def _new_heads(self, like, heads: int, n_tokens: int, other):
        """A tensor like `like` for a call to fill, and its description (as for _heads)."""
        out = self._like(like) if other is None else self._new(other, self._like, like)
        token, head, _ = out.stride()
        return out, smetric_heads(out.data_ptr(), token if n_tokens > 1 else 0, head if heads > 1 else 0)

    def _norm(self, w) -> Optional[int]:
        if w is None:
            return None
        if w.dtype != self.dtype or w.numel() != self._dim or not w.is_contiguous() or w.get_device() != self._device:
            raise ValueError(f"norm weights must be {self.dtype} [{self._dim}], contiguous, on cuda:{self._device}")
        return w.data_ptr()

    def _transform(self, cos_sin, interleaved, q_norm, k_norm, eps) -> smetric_kv_transform:
        rows = rot = table = None
        if cos_sin is not None:
            if (cos_sin.dtype != self._f32 or cos_sin.dim() != 2 or not cos_sin.is_contiguous() or
                    cos_sin.get_device() != self._device):
                raise ValueError(f"cos_sin must be torch.float32 [positions, rot_dim], contiguous, on cuda:{self._device}")
            rows, rot = cos_sin.shape
            # (a table without rows has no address, but NULL would say that there is no table: every token is
            # past its end, and no row is read)
            table = (cos_sin.data_ptr() if rows else 16) if rot else None
        return smetric_kv_transform(table, rows or 0, self._norm(q_norm), self._norm(k_norm), eps, rot or 0,
                                    SMETRIC_KV_INTERLEAVED if interleaved else 0, 0)

    def plan(self, offsets, kv_lens, pages, n_tokens: int, window: int = 0, stream=None, max_new: Optional[int] = None):
        """Plans a batch: offsets int64 [n+1], kv_lens int32 [n], pages int32
        [n, max_pages] (row stride free). The window is the plan's: layers that
        alternate need two plans or handles. max_new: no request has more new
        tokens (one that has is an error); steps of single tokens over caches in
        4 bits are faster when it says so. The handle keeps the tensors until
        the next plan, and until what read them on another stream than torch's
        current one at this call is done; those that a captured call reads are
        the graph's owner's to keep."""
        import torch
        n = kv_lens.numel()
        if offsets.dtype != torch.int64 or offsets.numel() != n + 1:
            raise ValueError("offsets must be torch.int64 [requests + 1]")
        if kv_lens.dtype != torch.int32 or pages.dtype != torch.int32 or pages.dim() != 2 or pages.shape[0] != n:
            raise ValueError("kv_lens must be torch.int32 [requests] and pages torch.int32 [requests, max_pages]")
        if any(x.get_device() != self._device for x in (offsets, kv_lens, pages)):
            raise ValueError(f"offsets, kv_lens and pages must be on cuda:{self._device}")
        if pages.shape[1] > 1 and pages.stride(1) != 1:
            raise ValueError("a request's pages must be contiguous")
        most = pages.shape[1]
        raw, other = self._stream(stream)
        args = (self.handle, offsets, n, n_tokens, kv_lens, pages.data_ptr() if pages.numel() else None, most,
                pages.stride(0) if n > 1 else most, max(-1 << 31, min(window, (1 << 31) - 1)))
        if max_new is None:
            smetric_kv_plan(*args, raw)
        else:
            smetric_kv_plan_up_to(*args, max(-1, min(max_new, (1 << 63) - 1)), raw)
        self._n_tokens = n_tokens
        self._keep((offsets, kv_lens, pages))
        self._read(raw, other)

    def _planned(self) -> int:
        if self._n_tokens is None:
            raise SmetricError(SMETRIC_ERR_INVALID_ARG, "no batch is planned")
        return self._n_tokens

    def append(self, k_cache, v_cache, k, v, q=None, q_out=None, cos_sin=None, interleaved=False, q_norm=None,
               k_norm=None, eps=1e-6, stream=None):
        """Appends the planned batch's keys (normed with k_norm, rotated with
        cos_sin where given) and values; with q, transforms the queries into
        q_out (a new tensor by default) and returns it."""
        t, c = self._planned(), self.cfg
        hk, hq = c.num_kv_heads, c.num_q_heads
        caches, kh, vh, qh = (self._caches(k_cache, v_cache), self._heads(k, hk, t, "k"), self._heads(v, hk, t, "v"),
                              self._heads(q, hq, t, "q"))
        raw, other = self._stream(stream)
        if q is None:
            q_out = None
        if q is not None and q_out is None:
            q_out, oh = self._new_heads(q, hq, t, other)
        else:
            oh = self._heads(q_out, hq, t, "q_out")
        _check(getattr(self._lib, self._append_call)(self.handle, *caches, kh, vh, qh, oh,
                                                     self._transform(cos_sin, interleaved, q_norm, k_norm, eps), raw),
               self._append_call)
        return q_out

    def qk_norm_rope(self, q, k, positions, cos_sin=None, interleaved=False, q_norm=None, k_norm=None, eps=1e-6,
                     q_out=None, k_out=None, stream=None):
        """The norms and the rotation alone, at int32 positions; q or k may be
        None. Returns (q_out, k_out), new tensors unless given."""
        t, c = positions.numel(), self.cfg
        if positions.dtype != self._i32 or not positions.is_contiguous() or positions.get_device() != self._device:
            raise ValueError(f"positions must be torch.int32, contiguous, on cuda:{self._device}")
        hk, hq = c.num_kv_heads, c.num_q_heads
        qh, kh = self._heads(q, hq, t, "q"), self._heads(k, hk, t, "k")
        raw, other = self._stream(stream)
        if q is None:
            q_out = None
        if k is None:
            k_out = None
        if q is not None and q_out is None:
            q_out, qo = self._new_heads(q, hq, t, other)
        else:
            qo = self._heads(q_out, hq, t, "q_out")
        if k is not None and k_out is None:
            k_out, ko = self._new_heads(k, hk, t, other)
        else:
            ko = self._heads(k_out, hk, t, "k_out")
        _check(self._lib.smetric_qk_norm_rope(self.handle, qh, kh, positions.data_ptr() if t else None, t,
                                              self._transform(cos_sin, interleaved, q_norm, k_norm, eps), qo, ko,
                                              raw), "smetric_qk_norm_rope")
        return q_out, k_out

    def paged_attention(self, q, k_cache, v_cache, scale=None, out=None, want_lse=False, stream=None):
        """Attention of the planned batch's queries over the cache; scale is
        head_dim ** -0.5 by default. Returns out, or (out, lse) with want_lse
        (float32 [tokens, num_q_heads])."""
        t, hq = self._planned(), self.cfg.num_q_heads
        caches, qh = self._caches(k_cache, v_cache), self._heads(q, hq, t, "q")
        raw, other = self._stream(stream)
        if out is None:
            out, oh = self._new_heads(q, hq, t, other)
        else:
            oh = self._heads(out, hq, t, "out")
        lse = self._new(other, self._empty, (t, hq), dtype=self._f32, device=q.device) if want_lse else None
        _check(getattr(self._lib, self._attention_call)(self.handle, *caches, qh,
                                                        self._dim ** -0.5 if scale is None else scale, oh,
                                                        lse.data_ptr() if want_lse and t else None, raw),
               self._attention_call)
        self._read(raw, other)
        return (out, lse) if want_lse else out

    def status(self, stream=None) -> int:
        return smetric_kv_status(self.handle, stream)

    def check(self, stream=None):
        rc = self.status(stream)
        if rc != SMETRIC_OK:
            raise SmetricError(rc, "device")


_NO_CACHE4 = smetric_kvq_cache()


class Cache4(NamedTuple):
    """Keys or values in 4 bits: codes uint8 [num_pages, page_size, num_kv_heads,
    head_dim / 2] and scales torch.float8_e4m3fn [num_pages, page_size,
    num_kv_heads, 4 (head_dim <= 64) or 8], views with any strides but the last;
    what they hold is code * scale * 2 ** exp."""

    codes: Any
    scales: Any
    exp: int = 0


class SMetricKV4(SMetricKV):
    """The paged KV$ operators with the caches in 4 bits (a scale of 8 bits for 16
    elements): SMetricKV's calls with a Cache4 for each cache, and read().

        kv = SMetricKV4(head_dim=128, num_q_heads=32, num_kv_heads=4, page_size=32, num_pages=16384,
                        max_batch_requests=64, max_batch_tokens=8192)
        cache = kv.new_cache()                                       # (keys, values)
        kv.plan(offsets_i64, kv_lens_i32, pages_i32, n_tokens)       # once a step
        kv.append(*cache, k, v, q=q, q_out=q, cos_sin=table, q_norm=wq, k_norm=wk)
        out = kv.paged_attention(q, *cache)
        k16, v16 = kv.read(*cache, rows_i64, pages_i32, n_rows)      # positions 0, 1, ... of every request
        kv.check()

    head_dim is a multiple of 32.
    """

    _flags = SMETRIC_KV_4BIT
    _append_call, _attention_call = "smetric_kvq_append", "smetric_kvq_attention"

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        import torch
        self._u8, self._e4m3, self._i64 = torch.uint8, torch.float8_e4m3fn, torch.int64
        rows = self._cache_shape[:3]
        self._codes_shape, self._scales_shape = rows + (self._dim // 2,), rows + (4 if self._dim <= 64 else 8,)

    def new_cache(self, k_exp: int = 0, v_exp: int = 0):
        """Caches for this handle: (keys, values), contiguous."""
        import torch
        make = lambda exp: Cache4(torch.zeros(self._codes_shape, dtype=self._u8, device=f"cuda:{self._device}"),  # noqa: E731
                                  torch.zeros(self._scales_shape, dtype=self._e4m3, device=f"cuda:{self._device}"), exp)
        return make(k_exp), make(v_exp)

    def _caches(self, k_cache, v_cache):
        return self._cache4(k_cache, "k_cache"), self._cache4(v_cache, "v_cache")

    def _cache4(self, cache, name: str) -> smetric_kvq_cache:
        if not isinstance(cache, Cache4):
            raise ValueError(f"{name} must be a Cache4")
        codes, scales, exp = cache
        here = self._device
        if (codes.dtype != self._u8 or scales.dtype != self._e4m3 or codes.shape != self._codes_shape or
                scales.shape != self._scales_shape or codes.get_device() != here or scales.get_device() != here):
            raise ValueError(f"{name}: codes must be {self._u8} {list(self._codes_shape)} and scales {self._e4m3} "
                             f"{list(self._scales_shape)}, on cuda:{here}")
        if not -SMETRIC_KVQ_MAX_EXP <= exp <= SMETRIC_KVQ_MAX_EXP:
            raise ValueError(f"{name}: exp must be within {SMETRIC_KVQ_MAX_EXP} of 0")
        p, t, h, one = codes.stride()
        sp, st, sh, sone = scales.stride()
        if one != 1 or sone != 1:
            raise ValueError(f"{name}: a head's codes and its scales must be contiguous")
        if self._cache_shape[0] == 1:  # (the stride of a dimension of one is arbitrary)
            p = sp = 0
        if self._cache_shape[2] == 1:
            h = sh = 0
        return smetric_kvq_cache(codes.data_ptr(), scales.data_ptr(), p, t, h, sp, st, sh, exp, 0)

    def read(self, k_cache, v_cache, offsets, pages, n_rows: int, first=None, k_out=None, v_out=None, stream=None):
        """What the caches hold: rows offsets[r]:offsets[r + 1] of the outputs get
        positions first[r], first[r] + 1, ... (0, 1, ... without first) of request
        r, in the handle's dtype. offsets int64 [n+1], first int32 [n], pages int32
        [n, max_pages] (row stride free). A cache may be None. Returns (k_out,
        v_out), new tensors [n_rows, num_kv_heads, head_dim] unless given; rows of
        no request are not written. offsets, pages and first may be dropped after
        the call, on another stream too; those that a captured call reads are the
        graph's owner's to keep."""
        hk, here, dim = self.cfg.num_kv_heads, self._device, self._dim
        n = offsets.numel() - 1
        if offsets.dtype != self._i64 or offsets.dim() != 1 or n < 0 or not offsets.is_contiguous():
            raise ValueError("offsets must be torch.int64 [requests + 1], contiguous")
        if pages.dtype != self._i32 or pages.dim() != 2:
            raise ValueError("pages must be torch.int32 [requests, max_pages]")
        (rows, most), (row_stride, one) = pages.shape, pages.stride()
        if rows != n or (most > 1 and one != 1):
            raise ValueError("pages must be torch.int32 [requests, max_pages], a request's contiguous")
        if first is not None and (first.dtype != self._i32 or first.shape != (n,) or not first.is_contiguous() or
                                  first.get_device() != here):
            raise ValueError(f"first must be torch.int32 [requests], contiguous, on cuda:{here}")
        if offsets.get_device() != here or pages.get_device() != here:
            raise ValueError(f"offsets and pages must be on cuda:{here}")
        raw, other = self._stream(stream)

        def out_of(cache, out, name):
            """A cache's description, its output and that one's description."""
            if cache is None:
                return _NO_CACHE4, None, _NO_HEADS
            described = self._cache4(cache, name)
            if out is not None:
                return described, out, self._heads(out, hk, n_rows, name)
            shape = (n_rows, hk, dim)
            out = (self._empty(shape, dtype=self.dtype, device=offsets.device) if other is None else
                   self._new(other, self._empty, shape, dtype=self.dtype, device=offsets.device))
            return described, out, smetric_heads(out.data_ptr(), hk * dim, dim)

        kc, k_out, kh = out_of(k_cache, k_out, "k")
        vc, v_out, vh = out_of(v_cache, v_out, "v")
        _check(self._lib.smetric_kvq_read(self.handle, kc, vc, offsets.data_ptr(), n, n_rows,
                                          first.data_ptr() if first is not None and n else None,
                                          pages.data_ptr() if n and most else None, most, row_stride if n > 1 else most,
                                          kh, vh, raw), "smetric_kvq_read")
        if other is not None:  # (torch may hand their memory out again only when that stream is done with them)
            for x in (offsets, pages) if first is None else (offsets, pages, first):
                x.record_stream(other)
        return k_out, v_out
