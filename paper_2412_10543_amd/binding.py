"""Thin Python binding of librag_attn.so (the C ABI in include/rag_attn.h).

Argument marshalling only: every step of the attention path runs in the HIP
library.  Tensors are torch tensors on the GPU (torch supplies device memory
and the current HIP stream); shapes, dtypes and contiguity are checked here
and everything else is left to the library's own validation.  There is no
fallback: if the library is missing or was built for another target, loading
raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

LIBRARY = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librag_attn.so")

RAG_NO_FIT = 1
RAG_OK = 0
RAG_ERR_INVALID_ARG = -1
RAG_ERR_UNSUPPORTED = -2
RAG_ERR_WORKSPACE = -3
RAG_ERR_HIP = -4

RAG_STUFF = 0
RAG_MAP_REDUCE_MAP = 1
RAG_MAP_REDUCE_REDUCE = 2
RAG_MAP_RERANK = 3
METHOD_CODES = {"stuff": RAG_STUFF, "map_reduce_map": RAG_MAP_REDUCE_MAP,
                "map_reduce_reduce": RAG_MAP_REDUCE_REDUCE, "map_rerank": RAG_MAP_RERANK}


class RagError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"rag_attn status {status}: {message}")
        self.status = status


_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_i32p = ctypes.POINTER(ctypes.c_int32)
_vp = ctypes.c_void_p
_lib = None
_marshal = None


def exported_symbols():
    return ["rag_abi_version", "rag_last_error", "rag_attn_prefill_varlen",
            "rag_attn_prefill_varlen_kvcache", "rag_attn_decode_paged_append",
            "rag_attn_decode_num_splits", "rag_attn_decode_workspace_size",
            "rag_attn_decode_paged", "rag_attn_decode_paged_noalloc", "rag_kv_cache_write", "rag_plan_prompts",
            "rag_prune_config_space", "rag_config_kv_bytes", "rag_choose_config",
            "rag_device_free_memory", "rag_awq_pack_weights", "rag_awq_workspace_size",
            "rag_awq_gemm", "rag_kv_pages_update", "rag_kv_cache_keep",
            "rag_attn_decode_tree_workspace_size", "rag_attn_decode_paged_tree",
            "rag_attn_prefill_varlen_ranges", "rag_qkv_rope_write", "rag_qkv_rope_write_kv4",
            "rag_kv4_read", "rag_attn_decode_kv4_workspace_size", "rag_attn_decode_paged_kv4",
            "rag_draft_verify_workspace_size", "rag_draft_verify"]


class QueryProfile(ctypes.Structure):
    _fields_ = [("complexity_high", ctypes.c_int32), ("joint_reasoning", ctypes.c_int32),
                ("pieces", ctypes.c_int32), ("summary_len_min", ctypes.c_int32),
                ("summary_len_max", ctypes.c_int32)]


class ConfigSpace(ctypes.Structure):
    _fields_ = [("methods", ctypes.c_uint32), ("num_chunks_min", ctypes.c_int32),
                ("num_chunks_max", ctypes.c_int32), ("intermediate_length_min", ctypes.c_int32),
                ("intermediate_length_max", ctypes.c_int32)]


class RequestShape(ctypes.Structure):
    _fields_ = [("query_len", ctypes.c_int32), ("chunk_len", ctypes.c_int32),
                ("answer_len", ctypes.c_int32), ("kv_bytes_per_token", ctypes.c_int64)]


class Config(ctypes.Structure):
    _fields_ = [("method", ctypes.c_int32), ("num_chunks", ctypes.c_int32),
                ("intermediate_length", ctypes.c_int32), ("fallback", ctypes.c_int32),
                ("kv_bytes", ctypes.c_int64)]


def lib():
    """Load (once) and return the ctypes handle of librag_attn.so."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIBRARY):
        raise ImportError(f"{LIBRARY} is not built; run __graft_entry__.build() or "
                          "python -m paper_2412_10543_amd.build")
    L = ctypes.CDLL(LIBRARY)
    L.rag_abi_version.restype = ctypes.c_int
    L.rag_last_error.restype = ctypes.c_char_p
    L.rag_attn_prefill_varlen.restype = ctypes.c_int
    L.rag_attn_prefill_varlen.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                                          _i32, _i32, _i32, ctypes.c_float, _i32, _vp]
    L.rag_attn_prefill_varlen_kvcache.restype = ctypes.c_int
    L.rag_attn_prefill_varlen_kvcache.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                                                  _i32, _i32, ctypes.c_float, _vp, _vp, _vp,
                                                  _i32, _i32, _vp]
    L.rag_attn_decode_paged_append.restype = ctypes.c_int
    L.rag_attn_decode_paged_append.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32,
                                               _i32, _i32, _i32, _i32, _i32, ctypes.c_float,
                                               _i32, _vp, ctypes.c_size_t, _vp]
    L.rag_attn_decode_num_splits.restype = _i32
    L.rag_attn_decode_num_splits.argtypes = [_i32, _i32, _i32, _i32, _i32]
    L.rag_attn_decode_workspace_size.restype = ctypes.c_size_t
    L.rag_attn_decode_workspace_size.argtypes = [_i32, _i32, _i32, _i32, _i32, _i32, _i32]
    L.rag_attn_decode_paged.restype = ctypes.c_int
    L.rag_attn_decode_paged.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                                        _i32, _i32, _i32, _i32, _i32, _i32, ctypes.c_float,
                                        _i32, _vp, ctypes.c_size_t, _vp]
    L.rag_attn_decode_paged_noalloc.restype = ctypes.c_int
    L.rag_attn_decode_paged_noalloc.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32,
                                                _i32, _i32, _i32, _i32, _i32, _i32, _i32,
                                                ctypes.c_float, _i32, _vp]
    L.rag_kv_cache_write.restype = ctypes.c_int
    L.rag_kv_cache_write.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _vp]
    L.rag_prune_config_space.restype = ctypes.c_int
    L.rag_prune_config_space.argtypes = [ctypes.POINTER(QueryProfile), ctypes.POINTER(ConfigSpace)]
    L.rag_config_kv_bytes.restype = ctypes.c_int64
    L.rag_config_kv_bytes.argtypes = [_i32, _i32, _i32, ctypes.POINTER(RequestShape)]
    L.rag_choose_config.restype = ctypes.c_int
    L.rag_choose_config.argtypes = [ctypes.POINTER(QueryProfile), ctypes.POINTER(RequestShape),
                                    ctypes.c_int64, ctypes.POINTER(Config)]
    L.rag_device_free_memory.restype = ctypes.c_int
    L.rag_device_free_memory.argtypes = [ctypes.POINTER(ctypes.c_size_t),
                                         ctypes.POINTER(ctypes.c_size_t)]
    L.rag_awq_pack_weights.restype = ctypes.c_int
    L.rag_awq_pack_weights.argtypes = [_vp, _i32, _i32, _i32, _vp]
    L.rag_awq_workspace_size.restype = ctypes.c_size_t
    L.rag_awq_workspace_size.argtypes = [_i32, _i32, _i32, _i32]
    L.rag_awq_gemm.restype = ctypes.c_int
    L.rag_awq_gemm.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp,
                               ctypes.c_size_t, _vp]
    L.rag_kv_pages_update.restype = ctypes.c_int
    L.rag_kv_pages_update.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _vp,
                                      _vp, _vp, _vp, _vp, _vp]
    L.rag_kv_cache_keep.restype = ctypes.c_int
    L.rag_kv_cache_keep.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32,
                                    _i32, _i32, _vp]
    L.rag_attn_decode_tree_workspace_size.restype = ctypes.c_size_t
    L.rag_attn_decode_tree_workspace_size.argtypes = [_i32] * 8
    L.rag_attn_decode_paged_tree.restype = ctypes.c_int
    L.rag_attn_decode_paged_tree.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32,
                                             _i32, _i32, _i32, _i32, _i32, _i32, _i32,
                                             ctypes.c_float, _i32, _vp, ctypes.c_size_t, _vp]
    L.rag_attn_prefill_varlen_ranges.restype = ctypes.c_int
    L.rag_attn_prefill_varlen_ranges.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32,
                                                 _i32, _i32, _i32, _i32, _i32, ctypes.c_float, _vp]
    for call in (L.rag_qkv_rope_write, L.rag_qkv_rope_write_kv4):
        call.restype = ctypes.c_int
        call.argtypes = [_vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                         _i32, _i32, _i32, _vp, _vp, ctypes.c_float, _i32, _i32, _i32, _i32, _i32,
                         _i32, _vp]
    L.rag_kv4_read.restype = ctypes.c_int
    L.rag_kv4_read.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _i32,
                               _i32, _vp]
    L.rag_attn_decode_kv4_workspace_size.restype = ctypes.c_size_t
    L.rag_attn_decode_kv4_workspace_size.argtypes = [_i32] * 7
    L.rag_attn_decode_paged_kv4.restype = ctypes.c_int
    L.rag_attn_decode_paged_kv4.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                                            _i32, _i32, _i32, _i32, _i32, ctypes.c_float, _vp,
                                            ctypes.c_size_t, _vp]
    L.rag_draft_verify_workspace_size.restype = ctypes.c_size_t
    L.rag_draft_verify_workspace_size.argtypes = [_i32, _i32, _i32]
    L.rag_draft_verify.restype = ctypes.c_int
    L.rag_draft_verify.argtypes = [_vp, _i32, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                   _vp, _i32, _i32, _i32, _i32, _vp, ctypes.c_size_t, _vp]
    L.rag_plan_prompts.restype = ctypes.c_int
    L.rag_plan_prompts.argtypes = [ctypes.c_int, _i32, _i32p, _i32p, _i32, _i32, _i32, _i32p,
                                   _i32, _i32p, _i32p]
    _lib = L
    return L


def _check(status: int):
    if status != RAG_OK:
        raise RagError(status, lib().rag_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    # (the raw handle of the current stream: building a Stream object for it
    # costs about as much as the rest of a call's marshalling)
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _refuse(t, dtype, name, ndim):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions")


def _need(t, dtype, name, ndim=None):
    """t is a contiguous GPU tensor of this dtype (and rank): one test in the
    usual case, the first that fails named otherwise."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()
            and (ndim is None or t.ndim == ndim)):
        _refuse(t, dtype, name, ndim)


def rag_abi_version() -> int:
    return lib().rag_abi_version()


def rag_last_error() -> str:
    return lib().rag_last_error().decode()


def rag_attn_prefill_varlen(q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q,
                            max_seqlen_k, softmax_scale, causal=True, stream=None) -> None:
    """q, o [Tq, Hq, d]; k, v [Tk, Hkv, d] bf16; lse fp32 [Hq, Tq] or None;
    cu_seqlens_* int32 [S+1] on the GPU."""
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o, "o")):
        _need(t, torch.bfloat16, n, 3)
    _need(cu_seqlens_q, torch.int32, "cu_seqlens_q", 1)
    _need(cu_seqlens_k, torch.int32, "cu_seqlens_k", 1)
    if lse is not None:
        _need(lse, torch.float32, "lse", 2)
    _check(lib().rag_attn_prefill_varlen(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(cu_seqlens_q), _ptr(cu_seqlens_k),
        cu_seqlens_q.numel() - 1, int(max_seqlen_q), int(max_seqlen_k), q.shape[1], k.shape[1],
        q.shape[2], float(softmax_scale), int(bool(causal)), _stream(stream)))


def rag_attn_prefill_varlen_kvcache(q, k, v, o, lse, cu_seqlens, max_seqlen, softmax_scale,
                                    k_cache, v_cache, slot_mapping, stream=None) -> None:
    """Causal prompt prefill that also writes K/V into the paged cache.
    q, o [T, Hq, d]; k, v [T, Hkv, d] bf16; cu_seqlens int32 [S+1]; caches
    [num_blocks, Hkv, 16, d] bf16; slot_mapping int32 [T] (negative = skip)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o, "o")):
        _need(t, torch.bfloat16, n, 3)
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _need(t, torch.bfloat16, n, 4)
    _need(cu_seqlens, torch.int32, "cu_seqlens", 1)
    _need(slot_mapping, torch.int32, "slot_mapping", 1)
    if lse is not None:
        _need(lse, torch.float32, "lse", 2)
    _check(lib().rag_attn_prefill_varlen_kvcache(
        _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(cu_seqlens), cu_seqlens.shape[0] - 1,
        int(max_seqlen), q.shape[1], k.shape[1], q.shape[2], float(softmax_scale),
        _ptr(k_cache), _ptr(v_cache), _ptr(slot_mapping), k_cache.shape[0], k_cache.shape[2],
        _stream(stream)))


def rag_attn_decode_paged_append(q, k_new, v_new, k_cache, v_cache, o, block_tables, kv_lens,
                                 softmax_scale, num_splits=0, workspace=None, stream=None):
    """One decode step that appends each row's new token (k_new, v_new
    [S, Hkv, d]) to the cache at key kv_lens[s] - 1 and attends it."""
    for t, n in ((q, "q"), (o, "o"), (k_new, "k_new"), (v_new, "v_new")):
        _need(t, torch.bfloat16, n, 3)
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _need(t, torch.bfloat16, n, 4)
    _need(block_tables, torch.int32, "block_tables", 2)
    _need(kv_lens, torch.int32, "kv_lens", 1)
    ws_bytes = 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous GPU tensor")
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().rag_attn_decode_paged_append(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o),
        _ptr(block_tables), _ptr(kv_lens), block_tables.shape[0], block_tables.shape[1],
        k_cache.shape[0], q.shape[1], k_cache.shape[1], q.shape[2], k_cache.shape[2],
        float(softmax_scale), int(num_splits), _ptr(workspace), ws_bytes, _stream(stream)))


def rag_attn_decode_num_splits(num_decode_seqs, num_kv_heads, max_blocks_per_seq,
                               block_size=16, num_splits=0) -> int:
    return lib().rag_attn_decode_num_splits(num_decode_seqs, num_kv_heads, max_blocks_per_seq,
                                            block_size, num_splits)


def rag_attn_decode_workspace_size(num_decode_seqs, num_q_heads, num_kv_heads, head_dim,
                                   max_blocks_per_seq, block_size=16, num_splits=0) -> int:
    return lib().rag_attn_decode_workspace_size(num_decode_seqs, num_q_heads, num_kv_heads,
                                                head_dim, max_blocks_per_seq, block_size,
                                                num_splits)


def rag_attn_decode_paged(q, k_cache, v_cache, o, block_tables, kv_lens, softmax_scale,
                          cu_seqlens_q=None, num_decode_seqs=None, max_seqlen_q=1,
                          num_splits=0, workspace=None, stream=None) -> None:
    """q, o [Tq, Hq, d]; caches [num_blocks, Hkv, 16, d] bf16; block_tables
    int32 [S, max_blocks]; kv_lens int32 [S]; cu_seqlens_q int32 [S+1] or
    None; workspace a zero-initialised GPU tensor (torch.zeros, uint8) of
    rag_attn_decode_workspace_size bytes, or None when that size is 0."""
    for t, n in ((q, "q"), (o, "o")):
        _need(t, torch.bfloat16, n, 3)
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _need(t, torch.bfloat16, n, 4)
    _need(block_tables, torch.int32, "block_tables", 2)
    _need(kv_lens, torch.int32, "kv_lens", 1)
    if cu_seqlens_q is not None:
        _need(cu_seqlens_q, torch.int32, "cu_seqlens_q", 1)
    num_seqs = block_tables.shape[0]
    if num_decode_seqs is None:
        num_decode_seqs = num_seqs
    ws_bytes = 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous GPU tensor")
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().rag_attn_decode_paged(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(block_tables), _ptr(kv_lens),
        _ptr(cu_seqlens_q), num_seqs, int(num_decode_seqs), block_tables.shape[1],
        int(max_seqlen_q), k_cache.shape[0], q.shape[1], k_cache.shape[1], q.shape[2],
        k_cache.shape[2], float(softmax_scale), int(num_splits), _ptr(workspace), ws_bytes,
        _stream(stream)))


def rag_attn_decode_paged_noalloc(q, k_cache, v_cache, o, block_tables, kv_lens, softmax_scale,
                                  cu_seqlens_q=None, num_decode_seqs=None, max_seqlen_q=1,
                                  num_splits=0, stream=None) -> None:
    """rag_attn_decode_paged with the library's static scratch instead of a
    workspace (allocates nothing)."""
    for t, n in ((q, "q"), (o, "o")):
        _need(t, torch.bfloat16, n, 3)
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _need(t, torch.bfloat16, n, 4)
    _need(block_tables, torch.int32, "block_tables", 2)
    _need(kv_lens, torch.int32, "kv_lens", 1)
    if cu_seqlens_q is not None:
        _need(cu_seqlens_q, torch.int32, "cu_seqlens_q", 1)
    num_seqs = block_tables.shape[0]
    if num_decode_seqs is None:
        num_decode_seqs = num_seqs
    _check(lib().rag_attn_decode_paged_noalloc(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(block_tables), _ptr(kv_lens),
        _ptr(cu_seqlens_q), num_seqs, int(num_decode_seqs), block_tables.shape[1],
        int(max_seqlen_q), k_cache.shape[0], q.shape[1], k_cache.shape[1], q.shape[2],
        k_cache.shape[2], float(softmax_scale), int(num_splits), _stream(stream)))


def rag_kv_cache_write(k, v, k_cache, v_cache, slot_mapping, stream=None) -> None:
    """k, v [T, Hkv, d] bf16; caches [num_blocks, Hkv, 16, d] bf16; slot_mapping
    int32 [T] on the GPU (negative = skip)."""
    for t, n in ((k, "k"), (v, "v")):
        _need(t, torch.bfloat16, n, 3)
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _need(t, torch.bfloat16, n, 4)
    _need(slot_mapping, torch.int32, "slot_mapping", 1)
    _check(lib().rag_kv_cache_write(
        _ptr(k), _ptr(v), _ptr(k_cache), _ptr(v_cache), _ptr(slot_mapping), k.shape[0],
        k.shape[1], k.shape[2], k_cache.shape[2], k_cache.shape[0], _stream(stream)))


def _pointers(spec, *tensors):
    """(device, address and sizes of each tensor) of contiguous tensors on the
    current device, with the types and ranks of spec (see csrc/marshal.cpp), or a
    number for _refuse_at."""
    if _marshal is None:
        _load_marshal()
    return _marshal.pointers(spec, *tensors)


def _load_marshal():
    """The library, and the native checks of tensors beside it."""
    global _marshal
    lib()
    try:
        from . import _marshal as loaded
    except ImportError as e:
        raise ImportError("_marshal.so is not built, or for another torch; run "
                          f"__graft_entry__.build() or python -m paper_2412_10543_amd.build ({e})") from e
    _marshal = loaded


_TYPES = {"i": torch.int32, "l": torch.int64, "u": torch.uint8, "b": torch.bfloat16,
          "f": torch.float32, "r": torch.bfloat16, "g": torch.float32}


def _refuse_at(i, spec, names, tensors):
    """Why tensor i was not taken."""
    first = next((t for t in tensors if isinstance(t, torch.Tensor)), None)   # (None: i's type is why)
    if i == len(tensors):
        raise ValueError(f"tensors on {first.device}, not on the current device")
    t, name, kind = tensors[i], names.split()[i], chr(spec[2 * i]).lower()
    rank = spec[2 * i + 1] - ord("0")
    if kind in "rgh" and isinstance(t, torch.Tensor):
        if kind == "h" and t.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"{name} must be bfloat16 or float32, got {t.dtype}")
        if t.dim() == rank and t.is_cuda and t.dtype == _TYPES.get(kind, t.dtype) and \
                first.device == t.device:
            raise ValueError(f"{name} must be contiguous but for the step from row to row, of at "
                             f"least a row; its strides are {tuple(t.stride())}")
        _refuse(t[:0].contiguous() if t.dim() else t, _TYPES.get(kind, t.dtype), name, rank)
    else:
        _refuse(t, _TYPES.get(kind, torch.bfloat16), name, rank)
    raise ValueError(f"{name} is on {t.device}, not on {first.device}")


def _scratch(workspace, dev):
    """(address, bytes) of a call's workspace tensor, or of None."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the current device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _raw_stream(stream, dev):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def rag_kv_pages_update(block_tables, free_pages, num_free, old_lens, new_lens, num_free_out,
                        lens_out, cu_new, slot_mapping, num_granted, stream=None) -> None:
    """Pages of S rows that hold old_lens tokens and are to hold new_lens: all
    int32 on the GPU; block_tables [S, max_blocks] and free_pages [num_blocks]
    in and out; num_free, num_free_out and num_granted [1]; lens_out [S],
    cu_new [S+1] and slot_mapping [max_new_tokens] outputs."""
    t = (block_tables, free_pages, num_free, old_lens, new_lens, num_free_out, lens_out, cu_new,
         slot_mapping, num_granted)
    p = _pointers(b"i2i1i1i1i1i1i1i1i1i1", *t)
    if p.__class__ is int:
        _refuse_at(p, b"i2i1i1i1i1i1i1i1i1i1", "block_tables free_pages num_free old_lens new_lens "
                   "num_free_out lens_out cu_new slot_mapping num_granted", t)
    dev, table, S, width, pages, blocks, free, one, old, rows, new, rows2, free_out, one2, lens, rows3, \
        cu, rows1, slots, tokens, granted, one3 = p
    if not (rows == rows2 == rows3 == rows1 - 1 == S and one == one2 == one3 == 1):
        raise ValueError("kv pages: inconsistent shapes")
    status = _lib.rag_kv_pages_update(table, pages, free, old, new, S, width, blocks, 16, tokens,
                                      free_out, lens, cu, slots, granted, _raw_stream(stream, dev))
    if status:
        _check(status)


def rag_kv_cache_keep(k_cache, v_cache, block_tables, base_lens, kept, num_kept,
                      stream=None) -> None:
    """Moves the K/V rows of the accepted drafted nodes behind their sequence's
    base_lens keys.  Caches [num_blocks, Hkv, 16, d] bf16; block_tables int32
    [S, max_blocks]; base_lens and num_kept int32 [S]; kept int32 [S, max_kept]."""
    t = (k_cache, v_cache, block_tables, kept, base_lens, num_kept)
    p = _pointers(b"b4b4i2i2i1i1", *t)
    if p.__class__ is int:
        _refuse_at(p, b"b4b4i2i2i1i1", "k_cache v_cache block_tables kept base_lens num_kept", t)
    dev, kc, blocks, hkv, block, d, vc, b2, h2, s2, d2, table, S, width, nodes, rows, max_kept, base, \
        rows2, num, rows3 = p
    if not rows == rows2 == rows3 == S or (b2, h2, s2, d2) != (blocks, hkv, block, d):
        raise ValueError("kv keep: inconsistent shapes")
    status = _lib.rag_kv_cache_keep(kc, vc, table, base, nodes, num, S, width, max_kept, blocks, hkv,
                                    d, block, _raw_stream(stream, dev))
    if status:
        _check(status)


def rag_attn_decode_tree_workspace_size(num_seqs, max_nodes, num_q_heads, num_kv_heads, head_dim,
                                        max_blocks_per_seq, block_size=16, num_splits=0) -> int:
    return lib().rag_attn_decode_tree_workspace_size(num_seqs, max_nodes, num_q_heads,
                                                     num_kv_heads, head_dim, max_blocks_per_seq,
                                                     block_size, num_splits)


def rag_attn_decode_paged_tree(q, k_cache, v_cache, o, tree_mask, block_tables, kv_lens,
                               cu_seqlens_q, max_nodes, softmax_scale, num_splits=0,
                               workspace=None, stream=None) -> None:
    """q, o [Tq, Hq, d]; caches [num_blocks, Hkv, 16, d] bf16; tree_mask int64
    [Tq, words]: bit j of row i's words set where node i sees node j; block_tables
    int32 [S, max_blocks]; kv_lens int32 [S], the nodes counted; cu_seqlens_q int32
    [S+1] offsets of the nodes; workspace a GPU tensor (torch.empty, uint8) of
    rag_attn_decode_tree_workspace_size bytes, or None when that size is 0."""
    t = (q, o, k_cache, v_cache, tree_mask, block_tables, kv_lens, cu_seqlens_q)
    p = _pointers(b"b3b3b4b4l2i2i1i1", *t)
    if p.__class__ is int:
        _refuse_at(p, b"b3b3b4b4l2i2i1i1", "q o k_cache v_cache tree_mask block_tables kv_lens "
                   "cu_seqlens_q", t)
    dev, qp, rows, hq, dq, op, rows2, hq2, dq2, kc, blocks, hkv, block, d, vc, b2, h2, s2, d2, mask, \
        rows3, words, table, S, width, kv, seqs, cu, seqs1 = p
    if (rows2, hq2, dq2) != (rows, hq, dq) or (b2, h2, s2, d2) != (blocks, hkv, block, d) or \
            dq != d or rows3 != rows or not seqs == seqs1 - 1 == S:
        raise ValueError("decode tree: inconsistent shapes")
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the current device")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if rows == 0:
        return
    status = _lib.rag_attn_decode_paged_tree(
        qp, kc, vc, op, mask, table, kv, cu, S, int(max_nodes), words, width, blocks, hq, hkv, d,
        block, float(softmax_scale), int(num_splits), ws_ptr, ws_bytes, _raw_stream(stream, dev))
    if status:
        _check(status)


def rag_attn_prefill_varlen_ranges(q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, key_ranges,
                                   max_seqlen_q, max_seqlen_k, softmax_scale, stream=None) -> None:
    """q, o [Tq, Hq, d]; k, v [Tk, Hkv, d] bf16; lse fp32 [Hq, cu_seqlens_q[-1]] or
    None (q and o may have rows behind those, lse not); cu_seqlens_* int32 [S+1];
    key_ranges int32 [Tq, 2]: the (shared, start) of each row, which sees the keys
    j < shared and start <= j <= its position."""
    t = (q, k, v, o, cu_seqlens_q, cu_seqlens_k, key_ranges, lse)
    p = _pointers(b"b3b3b3b3i1i1i2F2", *t)
    if p.__class__ is int:
        _refuse_at(p, b"b3b3b3b3i1i1i2F2", "q k v o cu_seqlens_q cu_seqlens_k key_ranges lse", t)
    dev, qp, rows, hq, d, kp, keys, hkv, dk, vp, keys2, hkv2, dv, op, rows2, hq2, d2, cu_q, seqs1, \
        cu_k, seqs2, ranges, rows3, two, lse_p = p[:25]
    if (rows2, hq2, d2) != (rows, hq, d) or (keys2, hkv2, dv) != (keys, hkv, d) or dk != d or \
            seqs1 != seqs2 or (rows3, two) != (rows, 2) or \
            (lse_p and (p[25] != hq or p[26] > rows)):
        raise ValueError("prefill ranges: inconsistent shapes")
    if rows == 0:
        return
    status = _lib.rag_attn_prefill_varlen_ranges(
        qp, kp, vp, op, lse_p, cu_q, cu_k, ranges, seqs1 - 1, int(max_seqlen_q), int(max_seqlen_k),
        hq, hkv, d, float(softmax_scale), _raw_stream(stream, dev))
    if status:
        _check(status)


def _rope_write(call, cache, q, k, v, q_out, positions, cos_sin, slot_mapping, k_cache, v_cache, k_out,
                v_out, q_weight, k_weight, eps, interleaved, stream):
    """`cache`: the spec of the caches, of which None gives zeros throughout."""
    t = (k, v, q, q_out, positions, cos_sin, slot_mapping, k_out, v_out, q_weight, k_weight, k_cache,
         v_cache)
    spec = b"r3r3R3B3I1F2I1B3B3B1B1" + cache
    p = _pointers(spec, *t)
    if p.__class__ is int:
        _refuse_at(p, spec, "k v q q_out positions cos_sin slot_mapping k_out v_out q_weight k_weight "
                   "k_cache v_cache", t)
    dev, kp, T, hkv, d, ks, vp, T2, hkv2, d2, vs, qp, T3, hq, d3, qs, qo, T4, hq4, d4, pos, T5, angles, \
        most, rot, slots, T6, ko, T7, h7, d7, vo, T8, h8, d8, qw, wq, kw, wk = p[:39]
    half = len(p) + 39 >> 1
    kc, *pages = p[39:half]
    vc, *pages2 = p[half:]
    blocks = pages[0]
    want = [blocks, hkv, 16, d] if len(pages) == 4 else [blocks, hkv, 9 * d]
    if (T2, hkv2, d2) != (T, hkv, d) or (q is not None and (T3, d3) != (T, d)) or \
            (q_out is not None and (T4, hq4, d4) != (T3, hq, d3)) or \
            (positions is not None and T5 != T) or (slot_mapping is not None and T6 != T) or \
            (k_out is not None and (T7, h7, d7) != (T, hkv, d)) or \
            (v_out is not None and (T8, h8, d8) != (T, hkv, d)) or \
            (q_weight is not None and wq != d) or (k_weight is not None and wk != d) or \
            (k_cache is not None and pages != want) or (v_cache is not None and pages2 != want):
        raise ValueError("qkv rope write: inconsistent shapes")
    status = getattr(_lib, call)(
        qp or None, kp, vp, qs, ks, vs, qo or None, ko or None, vo or None, kc or None, vc or None,
        slots or None, pos or None, angles or None, most, rot, 1 if interleaved else 0, qw or None,
        kw or None, float(eps), T, hq, hkv, d, 16, blocks, _raw_stream(stream, dev))
    if status:
        _check(status)


def rag_qkv_rope_write(q, k, v, q_out, positions, cos_sin, slot_mapping=None, k_cache=None,
                       v_cache=None, k_out=None, v_out=None, q_weight=None, k_weight=None, eps=1e-6,
                       interleaved=False, stream=None) -> None:
    """Norm of each head of Q and K, rotation, and the paged cache's write.  q
    [T, Hq, d] and k, v [T, Hkv, d] bf16, contiguous but for the step from token to
    token; q_out [T, Hq, d] (q and q_out None: K and V alone); positions int32 [T] and
    cos_sin fp32 [max_position, rotary_dim], or None (no rotation); slot_mapping int32
    [T] (negative = padding) and caches [num_blocks, Hkv, 16, d] bf16, or None; k_out,
    v_out [T, Hkv, d] or None; q_weight, k_weight bf16 [d] or None (no norm)."""
    _rope_write("rag_qkv_rope_write", b"B4B4", q, k, v, q_out, positions, cos_sin, slot_mapping,
                k_cache, v_cache, k_out, v_out, q_weight, k_weight, eps, interleaved, stream)


def rag_qkv_rope_write_kv4(q, k, v, q_out, positions, cos_sin, slot_mapping, k_cache, v_cache,
                           k_out=None, v_out=None, q_weight=None, k_weight=None, eps=1e-6,
                           interleaved=False, stream=None) -> None:
    """rag_qkv_rope_write into a 4-bit paged cache: k_cache, v_cache uint8
    [num_blocks, Hkv, 9 * d], slot_mapping int32 [T]."""
    _rope_write("rag_qkv_rope_write_kv4", b"U3U3", q, k, v, q_out, positions, cos_sin, slot_mapping,
                k_cache, v_cache, k_out, v_out, q_weight, k_weight, eps, interleaved, stream)


def rag_kv4_read(k_cache, v_cache, block_tables, cu_seqlens_k, k, v, stream=None) -> None:
    """The first cu_seqlens_k[s+1] - cu_seqlens_k[s] keys of every sequence of a 4-bit
    cache (uint8 [num_blocks, Hkv, 9 * d]) as bf16 rows: k, v [T, Hkv, d] outputs (rows
    behind cu_seqlens_k[S] stay); block_tables int32 [S, max_blocks]; cu_seqlens_k
    int32 [S+1]."""
    t = (k_cache, v_cache, block_tables, cu_seqlens_k, k, v)
    p = _pointers(b"u3u3i2i1b3b3", *t)
    if p.__class__ is int:
        _refuse_at(p, b"u3u3i2i1b3b3", "k_cache v_cache block_tables cu_seqlens_k k v", t)
    dev, kc, blocks, hkv, page, vc, b2, h2, p2, table, S, width, cu, seqs1, kp, T, hkv3, d, vp, T2, hkv4, \
        d2 = p
    if (b2, h2, p2) != (blocks, hkv, page) or (T2, hkv4, d2) != (T, hkv3, d) or hkv3 != hkv or \
            page != 9 * d or S != seqs1 - 1:
        raise ValueError("kv4 read: inconsistent shapes")
    status = _lib.rag_kv4_read(kc, vc, table, cu, kp, vp, T, S, width, blocks, hkv, d, 16,
                               _raw_stream(stream, dev))
    if status:
        _check(status)


def rag_attn_decode_kv4_workspace_size(num_seqs, max_seqlen_q, num_q_heads, num_kv_heads, head_dim,
                                       max_blocks_per_seq, block_size=16) -> int:
    return lib().rag_attn_decode_kv4_workspace_size(num_seqs, max_seqlen_q, num_q_heads, num_kv_heads,
                                                    head_dim, max_blocks_per_seq, block_size)


def rag_attn_decode_paged_kv4(q, k_cache, v_cache, o, block_tables, kv_lens, softmax_scale,
                              cu_seqlens_q=None, max_seqlen_q=None, workspace=None,
                              stream=None) -> None:
    """q, o [Tq, Hq, d] bf16; caches uint8 [num_blocks, Hkv, 9 * d]; block_tables int32
    [S, max_blocks]; kv_lens int32 [S], the rows counted; cu_seqlens_q int32 [S+1]
    offsets of the sequences' last rows, with max_seqlen_q, the most that one has, or
    None: one row each; workspace a GPU tensor of rag_attn_decode_kv4_workspace_size
    bytes, zero-filled once before its first use."""
    if max_seqlen_q is None:
        if cu_seqlens_q is not None:
            raise ValueError("decode kv4: cu_seqlens_q without max_seqlen_q")
        max_seqlen_q = 1
    t = (q, o, k_cache, v_cache, block_tables, kv_lens, cu_seqlens_q)
    p = _pointers(b"b3b3u3u3i2i1I1", *t)
    if p.__class__ is int:
        _refuse_at(p, b"b3b3u3u3i2i1I1", "q o k_cache v_cache block_tables kv_lens cu_seqlens_q", t)
    dev, qp, rows, hq, d, op, rows2, hq2, d2, kc, blocks, hkv, page, vc, b2, h2, p2, table, S, width, kv, \
        seqs, cu, seqs1 = p
    if (rows2, hq2, d2) != (rows, hq, d) or (b2, h2, p2) != (blocks, hkv, page) or page != 9 * d or \
            S != seqs or (rows if cu_seqlens_q is None else seqs1 - 1) != S:
        raise ValueError("decode kv4: inconsistent shapes")
    ws_ptr, ws_bytes = _scratch(workspace, dev)
    if rows == 0:
        return
    status = _lib.rag_attn_decode_paged_kv4(
        qp, kc, vc, op, table, kv, cu or None, S, int(max_seqlen_q), width, blocks, hq, hkv, d, 16,
        float(softmax_scale), ws_ptr, ws_bytes, _raw_stream(stream, dev))
    if status:
        _check(status)


def rag_draft_verify_workspace_size(num_rows, num_seqs, vocab) -> int:
    return lib().rag_draft_verify_workspace_size(num_rows, num_seqs, vocab)


def rag_draft_verify(logits, tokens, cu_seqlens_q, temperature, uniforms, kept, num_kept, next_token,
                     parents=None, draft_probs=None, workspace=None, stream=None) -> None:
    """logits [Tq, V] bf16 or fp32 and draft_probs fp32 [Tq, V] or None, contiguous but
    for the step from row to row; tokens int32 [Tq]; parents int32 [Tq] or None (chains);
    cu_seqlens_q int32 [S+1]; temperature fp32 [S]; uniforms fp32 [Tq]; kept int32
    [S, max_kept], num_kept and next_token int32 [S] outputs; workspace a GPU tensor of
    rag_draft_verify_workspace_size bytes, zero-filled once before its first use."""
    t = (logits, tokens, cu_seqlens_q, temperature, uniforms, kept, num_kept, next_token, parents,
         draft_probs)
    p = _pointers(b"h2i1i1f1f1i2i1i1I1G2", *t)
    if p.__class__ is int:
        _refuse_at(p, b"h2i1i1f1f1i2i1i1I1G2", "logits tokens cu_seqlens_q temperature uniforms kept "
                   "num_kept next_token parents draft_probs", t)
    dev, lp, rows, vocab, step, wide, tok, rows2, cu, seqs1, heat, S, u, rows3, ke, S2, most, nk, S3, nt, S4, \
        par, rows4, draft, rows5, vocab2, dstep = p
    if not rows == rows2 == rows3 or not S == S2 == S3 == S4 == seqs1 - 1 or \
            (parents is not None and rows4 != rows) or \
            (draft_probs is not None and (rows5, vocab2) != (rows, vocab)):
        raise ValueError("draft verify: inconsistent shapes")
    ws_ptr, ws_bytes = _scratch(workspace, dev)
    status = _lib.rag_draft_verify(
        lp, wide, step, draft or None, dstep, tok, par or None, cu, heat, u, ke, nk, nt, rows, S, vocab,
        most, ws_ptr, ws_bytes, _raw_stream(stream, dev))
    if status:
        _check(status)


def rag_plan_prompts(method, query_len, num_chunks, chunk_len, intermediate_length=0,
                     answer_len=0):
    """Host planner.  Returns (cu_seqlens list, decode_len list)."""
    code = METHOD_CODES[method] if isinstance(method, str) else int(method)
    n = len(query_len)
    ql = (_i32 * max(n, 1))(*query_len)
    nc = (_i32 * max(n, 1))(*num_chunks)
    count = _i32(0)
    L = lib()
    st = L.rag_plan_prompts(code, n, ql, nc, chunk_len, intermediate_length, answer_len, None, 0,
                            ctypes.byref(count), None)
    if st not in (RAG_OK, RAG_ERR_WORKSPACE):
        _check(st)
    cap = count.value + 1
    cu = (_i32 * cap)()
    dec = (_i32 * max(count.value, 1))()
    _check(L.rag_plan_prompts(code, n, ql, nc, chunk_len, intermediate_length, answer_len, cu,
                              cap, ctypes.byref(count), dec))
    return list(cu), list(dec)[:count.value]


# ---------------------------------------------------------------------------
# configuration planner (host only)
# ---------------------------------------------------------------------------
CONFIG_METHOD_NAMES = {RAG_STUFF: "stuff", RAG_MAP_REDUCE_MAP: "map_reduce",
                       RAG_MAP_RERANK: "map_rerank"}


def _profile(complexity_high, joint_reasoning, pieces, summary_range):
    return QueryProfile(int(bool(complexity_high)), int(bool(joint_reasoning)), int(pieces),
                        int(summary_range[0]), int(summary_range[1]))


def rag_prune_config_space(complexity_high, joint_reasoning, pieces, summary_range):
    """Algorithm 1.  Returns (method names, (chunks_min, chunks_max),
    (il_min, il_max))."""
    sp = ConfigSpace()
    _check(lib().rag_prune_config_space(
        ctypes.byref(_profile(complexity_high, joint_reasoning, pieces, summary_range)),
        ctypes.byref(sp)))
    methods = tuple(n for m, n in CONFIG_METHOD_NAMES.items() if sp.methods & (1 << m))
    return methods, (sp.num_chunks_min, sp.num_chunks_max), \
        (sp.intermediate_length_min, sp.intermediate_length_max)


def _shape(query_len, chunk_len, answer_len, bytes_per_token):
    return RequestShape(int(query_len), int(chunk_len), int(answer_len), int(bytes_per_token))


def rag_config_kv_bytes(method, num_chunks, intermediate_length, query_len, chunk_len,
                        answer_len, bytes_per_token) -> int:
    code = {v: k for k, v in CONFIG_METHOD_NAMES.items()}[method] if isinstance(method, str) \
        else int(method)
    return lib().rag_config_kv_bytes(code, int(num_chunks), int(intermediate_length),
                                     ctypes.byref(_shape(query_len, chunk_len, answer_len,
                                                         bytes_per_token)))


def rag_choose_config(complexity_high, joint_reasoning, pieces, summary_range, query_len,
                      chunk_len, answer_len, bytes_per_token, available_bytes):
    """Best-fit choice.  Returns a dict (method name, num_chunks,
    intermediate_length, kv_bytes, fallback) or None when nothing fits."""
    out = Config()
    st = lib().rag_choose_config(
        ctypes.byref(_profile(complexity_high, joint_reasoning, pieces, summary_range)),
        ctypes.byref(_shape(query_len, chunk_len, answer_len, bytes_per_token)),
        int(available_bytes), ctypes.byref(out))
    if st == RAG_NO_FIT:
        return None
    _check(st)
    return dict(method=CONFIG_METHOD_NAMES[out.method], num_chunks=out.num_chunks,
                intermediate_length=out.intermediate_length, kv_bytes=out.kv_bytes,
                fallback=bool(out.fallback))


def rag_device_free_memory():
    """(free bytes, total bytes) of the current HIP device."""
    f, t = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().rag_device_free_memory(ctypes.byref(f), ctypes.byref(t)))
    return f.value, t.value


def rag_awq_pack_weights(q, group_size: int = 128):
    """Host packer: q a numpy uint8 array [K, N] of 4-bit codes -> numpy int32
    [K // group_size, N, 16] in the kernel's order."""
    import numpy as np
    q = np.ascontiguousarray(q, dtype=np.uint8)
    if q.ndim != 2:
        raise ValueError("q must be [K, N]")
    K, N = q.shape
    out = np.empty((max(K // 128, 0), N, 16), dtype=np.int32)
    _check(lib().rag_awq_pack_weights(q.ctypes.data, K, N, int(group_size), out.ctypes.data))
    return out


def rag_awq_workspace_size(M: int, N: int, K: int, group_size: int = 128) -> int:
    return int(lib().rag_awq_workspace_size(int(M), int(N), int(K), int(group_size)))


def rag_awq_gemm(x, qweight, scales, zeros, y, workspace, group_size: int = 128,
                 stream=None) -> None:
    """x [M, K] bf16; qweight int32 [K/128, N, 16] (rag_awq_pack_weights);
    scales bf16 [K/128, N]; zeros uint8 [K/128, N]; y [M, N] bf16 output;
    workspace a GPU uint8 tensor of rag_awq_workspace_size bytes, zero-filled
    once before its first use (every call leaves its counters zero again)."""
    _need(x, torch.bfloat16, "x", 2)
    _need(qweight, torch.int32, "qweight", 3)
    _need(scales, torch.bfloat16, "scales", 2)
    _need(zeros, torch.uint8, "zeros", 2)
    _need(y, torch.bfloat16, "y", 2)
    M, K = x.shape
    N = y.shape[1]
    if y.shape[0] != M or qweight.shape != (K // 128, N, 16) or \
            scales.shape != (K // 128, N) or zeros.shape != (K // 128, N):
        raise ValueError("awq gemm: inconsistent shapes")
    ws_bytes = 0
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous GPU tensor")
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().rag_awq_gemm(_ptr(x), _ptr(qweight), _ptr(scales), _ptr(zeros), _ptr(y), M, N,
                              K, int(group_size), _ptr(workspace), ws_bytes, _stream(stream)))
