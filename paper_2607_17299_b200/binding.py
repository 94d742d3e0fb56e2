"""Thin Python binding of libwar.so: argument marshalling only.

Every function here has the name and the meaning of the C entry point it wraps (see include/war.h); tensors are
torch CUDA tensors used as device buffers, and the current torch stream is the stream of the call.  Nothing is
computed on the Python side, and there is no fallback: if the library has not been built, importing this module
raises."""
from __future__ import annotations

import ctypes as C
import functools
import math
import os
from typing import NamedTuple, Optional, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwar.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_17299_b200.build` "
                      "(there is no CPU or PyTorch fallback for this library)")
_lib = C.CDLL(LIB_PATH)

WAR_OK = 0
STATUS_NAMES = {0: "WAR_OK", 1: "WAR_ERR_INVALID_ARG", 2: "WAR_ERR_OOM", 3: "WAR_ERR_CAPACITY", 4: "WAR_ERR_CUDA",
                5: "WAR_ERR_TIMEOUT", 6: "WAR_ERR_UNSUPPORTED", 7: "WAR_ERR_BAD_TREE", 8: "WAR_ERR_BAD_PAGE"}

EXPORTS = ["war_index_build", "war_index_append", "war_index_append_async", "war_index_evict", "war_index_export_bytes", "war_index_export",
           "war_index_import", "war_index_info", "war_index_destroy", "war_draft", "war_draft_scored_workspace_bytes", "war_draft_scored", "war_draft_local", "war_draft_pick",
           "war_verify_attn_workspace_bytes", "war_verify_attn", "war_verify_attn_noalloc", "war_accept", "war_commit", "war_device_status",
           "war_rope_store", "war_rope_frequencies", "war_verify_attn_quant_workspace_bytes", "war_verify_attn_quant", "war_target",
           "war_commit_quant", "war_pages_grow", "war_pages_fork", "war_pages_free", "war_pages_compact_workspace_bytes", "war_pages_compact",
           "war_pages_copy", "war_prefix_groups", "war_verify_attn_shared_workspace_bytes", "war_verify_attn_shared",
           "war_verify_attn_shared_quant_workspace_bytes", "war_verify_attn_shared_quant",
           "war_selftest_bounded_wait",
           "war_status_string"]


class WarError(RuntimeError):
    def __init__(self, fn: str, code: int):
        self.code = code
        super().__init__(f"{fn} returned {STATUS_NAMES.get(code, code)}: {status_string(code)}")


class IndexInfo(C.Structure):
    _fields_ = [("M", C.c_int64), ("capacity_tokens", C.c_int64), ("T", C.c_int32), ("vocab", C.c_int32),
                ("max_depth", C.c_int32), ("reserved", C.c_int32), ("d_corpus", C.c_void_p), ("d_sa", C.c_void_p),
                ("d_lcp", C.c_void_p), ("d_bucket", C.c_void_p)]


class DraftParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("P", C.c_int32), ("N", C.c_int32), ("topk", C.c_int32), ("min_match", C.c_int32),
                ("spec_batch_limit", C.c_int32), ("spec_factor_num", C.c_int32), ("spec_factor_den", C.c_int32),
                ("min_prob_num", C.c_int32), ("min_prob_den", C.c_int32)]


class AttnParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("page_size", C.c_int32), ("max_pages_per_req", C.c_int32), ("kernel", C.c_int32),
                ("num_pages", C.c_int64), ("scale", C.c_float), ("reserved", C.c_int32),
                ("k_strides", C.c_int64 * 4), ("v_strides", C.c_int64 * 4)]


_lib.war_status_string.restype = C.c_char_p
_lib.war_status_string.argtypes = [C.c_int]
_lib.war_index_build.restype = C.c_int
_lib.war_index_build.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_void_p,
                                 C.POINTER(C.c_void_p)]
_lib.war_index_append.restype = C.c_int
_lib.war_index_append.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
_lib.war_index_append_async.restype = C.c_int
_lib.war_index_append_async.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
_lib.war_index_evict.restype = C.c_int
_lib.war_index_evict.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
_lib.war_index_export_bytes.restype = C.c_size_t
_lib.war_index_export_bytes.argtypes = [C.c_void_p]
_lib.war_index_export.restype = C.c_int
_lib.war_index_export.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.war_index_import.restype = C.c_int
_lib.war_index_import.argtypes = [C.c_void_p, C.c_size_t, C.c_int64, C.c_void_p, C.POINTER(C.c_void_p)]
_lib.war_index_info.restype = C.c_int
_lib.war_index_info.argtypes = [C.c_void_p, C.POINTER(IndexInfo)]
_lib.war_index_destroy.restype = C.c_int
_lib.war_index_destroy.argtypes = [C.c_void_p]
_lib.war_draft.restype = C.c_int
_lib.war_draft.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(DraftParams)] + [C.c_void_p] * 6
_lib.war_verify_attn_workspace_bytes.restype = C.c_size_t
_lib.war_draft_scored_workspace_bytes.restype = C.c_size_t
_lib.war_draft_scored_workspace_bytes.argtypes = [C.POINTER(DraftParams), C.c_int32]
_lib.war_draft_scored.restype = C.c_int
_lib.war_draft_scored.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(DraftParams), C.c_int32] + [C.c_void_p] * 8
_lib.war_draft_local.restype = C.c_int
_lib.war_draft_local.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(DraftParams)] + [C.c_void_p] * 6
_lib.war_draft_pick.restype = C.c_int
_lib.war_draft_pick.argtypes = [C.c_int32, C.c_int32] + [C.c_void_p] * 17
_lib.war_verify_attn_workspace_bytes.argtypes = [C.POINTER(AttnParams)]
_lib.war_verify_attn.restype = C.c_int
_lib.war_verify_attn.argtypes = [C.c_void_p] * 7 + [C.POINTER(AttnParams)] + [C.c_void_p] * 4
_lib.war_verify_attn_noalloc.restype = C.c_int
_lib.war_verify_attn_noalloc.argtypes = [C.c_void_p] * 7 + [C.POINTER(AttnParams)] + [C.c_void_p] * 3
_lib.war_accept.restype = C.c_int
_lib.war_accept.argtypes = [C.c_void_p] * 4 + [C.c_int32] * 3 + [C.c_void_p] * 4
_lib.war_device_status.restype = C.c_int
_lib.war_device_status.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]


def status_string(code: int) -> str:
    return _lib.war_status_string(int(code)).decode()


# (building a torch.cuda.Stream for every call takes 3 us of the host; the raw handle is the same)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor], dtype=None) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device buffers must be contiguous CUDA tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _check(fn: str, code: int) -> None:
    if code != WAR_OK:
        raise WarError(fn, code)


class Index:
    """Owner of a war_index_t*."""

    def __init__(self, handle: int):
        self._h = C.c_void_p(handle)

    @property
    def handle(self) -> C.c_void_p:
        if not self._h:
            raise ValueError("index already destroyed")
        return self._h

    def destroy(self) -> None:
        if self._h:
            _lib.war_index_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _offsets(h_offsets) -> np.ndarray:
    off = np.ascontiguousarray(np.asarray(h_offsets, dtype=np.int64))
    if off.ndim != 1 or len(off) < 1:
        raise ValueError("h_offsets must be int64 [T+1]")
    return off


def war_index_build(d_tokens: torch.Tensor, h_offsets, vocab: int, max_depth: int, capacity_tokens: int) -> Index:
    off = _offsets(h_offsets)
    out = C.c_void_p(None)
    code = _lib.war_index_build(_ptr(d_tokens, torch.int32), off.ctypes.data, len(off) - 1, vocab, max_depth,
                                capacity_tokens, _stream(), C.byref(out))
    _check("war_index_build", code)
    return Index(out.value)


def war_index_append(ix: Index, d_tokens: torch.Tensor, h_offsets) -> None:
    off = _offsets(h_offsets)
    _check("war_index_append", _lib.war_index_append(ix.handle, _ptr(d_tokens, torch.int32), off.ctypes.data,
                                                     len(off) - 1, _stream()))


def war_index_append_async(ix: Index, d_tokens: torch.Tensor, h_offsets) -> None:
    """Enqueues the append on the current stream and returns; keep d_tokens alive until that stream has run it."""
    off = _offsets(h_offsets)
    _check("war_index_append_async", _lib.war_index_append_async(ix.handle, _ptr(d_tokens, torch.int32), off.ctypes.data,
                                                                 len(off) - 1, _stream()))


def war_index_evict(ix: Index, n_oldest: int) -> None:
    _check("war_index_evict", _lib.war_index_evict(ix.handle, int(n_oldest), _stream()))


def war_index_export(ix: Index) -> np.ndarray:
    """The whole index as one host byte array (see war_index_import)."""
    n = int(_lib.war_index_export_bytes(ix.handle))
    buf = np.empty(n, dtype=np.uint8)
    _check("war_index_export", _lib.war_index_export(ix.handle, buf.ctypes.data, n, _stream()))
    return buf


def war_index_import(buf: np.ndarray, capacity_tokens: int) -> Index:
    buf = np.ascontiguousarray(buf, dtype=np.uint8)
    h = C.c_void_p()
    _check("war_index_import", _lib.war_index_import(buf.ctypes.data, buf.nbytes, int(capacity_tokens), _stream(), C.byref(h)))
    return Index(h.value)


def war_index_info(ix: Index) -> IndexInfo:
    info = IndexInfo()
    _check("war_index_info", _lib.war_index_info(ix.handle, C.byref(info)))
    return info


def war_index_destroy(ix: Index) -> None:
    ix.destroy()


def war_draft(ix: Index, d_tail: torch.Tensor, d_tail_len: torch.Tensor, N: int, topk: int, min_match: int,
              d_match_len: torch.Tensor, d_num_nodes: torch.Tensor, d_ids: torch.Tensor, d_parent: torch.Tensor,
              d_count: Optional[torch.Tensor], spec_batch_limit: int = 0, spec_factor=(0, 1), min_prob=(0, 1)) -> None:
    """spec_factor / min_prob are (numerator, denominator) pairs; a numerator of 0 switches the rule off."""
    B, P = d_tail.shape
    p = DraftParams(B, P, N, topk, min_match, spec_batch_limit, spec_factor[0], spec_factor[1], min_prob[0], min_prob[1])
    code = _lib.war_draft(ix.handle, _ptr(d_tail, torch.int32), _ptr(d_tail_len, torch.int32), C.byref(p),
                          _ptr(d_match_len, torch.int32), _ptr(d_num_nodes, torch.int32), _ptr(d_ids, torch.int32),
                          _ptr(d_parent, torch.int32), _ptr(d_count, torch.int32), _stream())
    _check("war_draft", code)


def war_draft_scored_workspace_bytes(B: int, P: int, N: int, topk: int, n_lengths: int) -> int:
    p = DraftParams(B, P, N, topk, 1, 0, 0, 1, 0, 1)
    return int(_lib.war_draft_scored_workspace_bytes(C.byref(p), n_lengths))


def war_draft_scored(ix: Index, d_tail: torch.Tensor, d_tail_len: torch.Tensor, N: int, topk: int, min_match: int,
                     n_lengths: int, d_workspace: torch.Tensor, d_match_len: torch.Tensor, d_used_len: torch.Tensor,
                     d_num_nodes: torch.Tensor, d_ids: torch.Tensor, d_parent: torch.Tensor, d_count: Optional[torch.Tensor],
                     spec_batch_limit: int = 0, spec_factor=(0, 1), min_prob=(0, 1)) -> None:
    """war_draft from the best-scoring of n_lengths suffix lengths; d_workspace is a uint8 CUDA tensor of at least
    war_draft_scored_workspace_bytes(...) bytes."""
    B, P = d_tail.shape
    p = DraftParams(B, P, N, topk, min_match, spec_batch_limit, spec_factor[0], spec_factor[1], min_prob[0], min_prob[1])
    need = int(_lib.war_draft_scored_workspace_bytes(C.byref(p), n_lengths))
    if need == 0 or d_workspace.dtype != torch.uint8 or not d_workspace.is_cuda or d_workspace.numel() < need:
        raise ValueError("workspace must be a uint8 CUDA tensor of war_draft_scored_workspace_bytes bytes")
    code = _lib.war_draft_scored(ix.handle, _ptr(d_tail, torch.int32), _ptr(d_tail_len, torch.int32), C.byref(p), n_lengths,
                                 d_workspace.data_ptr(), _ptr(d_match_len, torch.int32), _ptr(d_used_len, torch.int32),
                                 _ptr(d_num_nodes, torch.int32), _ptr(d_ids, torch.int32), _ptr(d_parent, torch.int32),
                                 _ptr(d_count, torch.int32), _stream())
    _check("war_draft_scored", code)


def war_draft_local(d_ctx: torch.Tensor, d_ctx_off: torch.Tensor, d_tail_len: torch.Tensor, P: int, N: int, topk: int,
                    min_match: int, d_match_len: torch.Tensor, d_num_nodes: torch.Tensor, d_ids: torch.Tensor,
                    d_parent: torch.Tensor, d_count: Optional[torch.Tensor], spec_batch_limit: int = 0, spec_factor=(0, 1),
                    min_prob=(0, 1)) -> None:
    """d_ctx: int32 tokens of all contexts back to back; d_ctx_off: int64 [B+1] bounds, both on the device."""
    B = d_ctx_off.numel() - 1
    p = DraftParams(B, P, N, topk, min_match, spec_batch_limit, spec_factor[0], spec_factor[1], min_prob[0], min_prob[1])
    code = _lib.war_draft_local(_ptr(d_ctx, torch.int32), _ptr(d_ctx_off, torch.int64), _ptr(d_tail_len, torch.int32),
                                C.byref(p), _ptr(d_match_len, torch.int32), _ptr(d_num_nodes, torch.int32),
                                _ptr(d_ids, torch.int32), _ptr(d_parent, torch.int32), _ptr(d_count, torch.int32), _stream())
    _check("war_draft_local", code)


def war_draft_pick(a, b, d_source: torch.Tensor, d_match_len: torch.Tensor, d_num_nodes: torch.Tensor, d_ids: torch.Tensor,
                   d_parent: torch.Tensor, d_count: Optional[torch.Tensor]) -> None:
    """a, b: (match_len, num_nodes, ids, parent, count) tensor tuples of the two trees."""
    B, N = a[2].shape
    args = [_ptr(t, torch.int32) for t in (*a, *b)]
    code = _lib.war_draft_pick(B, N, *args, _ptr(d_source, torch.int32), _ptr(d_match_len, torch.int32),
                               _ptr(d_num_nodes, torch.int32), _ptr(d_ids, torch.int32), _ptr(d_parent, torch.int32),
                               _ptr(d_count, torch.int32), _stream())
    _check("war_draft_pick", code)


def attn_params(q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, page_table: torch.Tensor, scale: float,
                kernel: int = 0) -> AttnParams:
    B, N, Hq, D = q.shape
    num_pages, Hkv, pg, _ = k_pool.shape
    p = AttnParams()
    p.B, p.N, p.Hq, p.Hkv, p.D, p.page_size = B, N, Hq, Hkv, D, pg
    p.max_pages_per_req = page_table.shape[1]
    p.kernel = kernel
    p.num_pages = num_pages
    p.scale = scale
    for i in range(4):
        p.k_strides[i] = k_pool.stride(i)
        p.v_strides[i] = v_pool.stride(i)
    return p


def war_verify_attn_workspace_bytes(params: AttnParams) -> int:
    return int(_lib.war_verify_attn_workspace_bytes(C.byref(params)))


def war_verify_attn(d_q: torch.Tensor, d_kpool: torch.Tensor, d_vpool: torch.Tensor, d_page_table: torch.Tensor,
                    d_prefix_len: torch.Tensor, d_num_nodes: torch.Tensor, d_parent: torch.Tensor, params: AttnParams,
                    d_workspace: torch.Tensor, d_out: torch.Tensor, d_lse: Optional[torch.Tensor]) -> None:
    for t in (d_kpool, d_vpool):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("pools must be bf16 CUDA tensors")
    code = _lib.war_verify_attn(_ptr(d_q, torch.bfloat16), d_kpool.data_ptr(), d_vpool.data_ptr(),
                                _ptr(d_page_table, torch.int32), _ptr(d_prefix_len, torch.int32),
                                _ptr(d_num_nodes, torch.int32), _ptr(d_parent, torch.int32), C.byref(params),
                                _ptr(d_workspace), _ptr(d_out, torch.bfloat16), _ptr(d_lse, torch.float32), _stream())
    _check("war_verify_attn", code)


NOALLOC_MAX_BYTES = 64 * 1024 * 1024


def war_verify_attn_noalloc(d_q: torch.Tensor, d_kpool: torch.Tensor, d_vpool: torch.Tensor, d_page_table: torch.Tensor,
                            d_prefix_len: torch.Tensor, d_num_nodes: torch.Tensor, d_parent: torch.Tensor,
                            params: AttnParams, d_out: torch.Tensor, d_lse: Optional[torch.Tensor]) -> None:
    """war_verify_attn without a workspace argument, for callers that cannot allocate device memory: the scratch
    is a fixed array inside the library (NOALLOC_MAX_BYTES).  Calls on one device share it, so keep them in stream
    order; make the first call on a device outside any stream capture."""
    for t in (d_kpool, d_vpool):
        if not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError("pools must be bf16 CUDA tensors")
    code = _lib.war_verify_attn_noalloc(_ptr(d_q, torch.bfloat16), d_kpool.data_ptr(), d_vpool.data_ptr(),
                                        _ptr(d_page_table, torch.int32), _ptr(d_prefix_len, torch.int32),
                                        _ptr(d_num_nodes, torch.int32), _ptr(d_parent, torch.int32), C.byref(params),
                                        _ptr(d_out, torch.bfloat16), _ptr(d_lse, torch.float32), _stream())
    _check("war_verify_attn_noalloc", code)


def war_accept(d_ids: torch.Tensor, d_parent: torch.Tensor, d_num_nodes: torch.Tensor, d_target_ids: torch.Tensor,
               target_mode: int, d_accept_len: torch.Tensor, d_accept_path: torch.Tensor, d_bonus: torch.Tensor) -> None:
    B, N = d_ids.shape
    code = _lib.war_accept(_ptr(d_ids, torch.int32), _ptr(d_parent, torch.int32), _ptr(d_num_nodes, torch.int32),
                           _ptr(d_target_ids, torch.int32), B, N, target_mode, _ptr(d_accept_len, torch.int32),
                           _ptr(d_accept_path, torch.int32), _ptr(d_bonus, torch.int32), _stream())
    _check("war_accept", code)


class CommitParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("P", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("page_size", C.c_int32), ("max_pages_per_req", C.c_int32), ("reserved", C.c_int32),
                ("num_pages", C.c_int64), ("k_strides", C.c_int64 * 4), ("v_strides", C.c_int64 * 4)]


_lib.war_commit.restype = C.c_int
_lib.war_commit.argtypes = [C.c_void_p] * 7 + [C.POINTER(CommitParams)] + [C.c_void_p] * 4


def war_commit(d_ids: torch.Tensor, d_accept_len: torch.Tensor, d_accept_path: torch.Tensor, d_bonus: torch.Tensor,
               k_pool: torch.Tensor, v_pool: torch.Tensor, page_table: torch.Tensor, d_prefix_len: torch.Tensor,
               d_tail: torch.Tensor, d_tail_len: torch.Tensor) -> None:
    """Pools are [pages, Hkv, page_size, D] bf16 views (any strides the library accepts); updated in place."""
    B, N = d_ids.shape
    p = CommitParams()
    p.B, p.N, p.P = B, N, d_tail.shape[1]
    p.Hkv, p.D, p.page_size = k_pool.shape[1], k_pool.shape[3], k_pool.shape[2]
    p.max_pages_per_req, p.num_pages = page_table.shape[1], k_pool.shape[0]
    for i in range(4):
        p.k_strides[i] = k_pool.stride(i)
        p.v_strides[i] = v_pool.stride(i)
    code = _lib.war_commit(_ptr(d_ids, torch.int32), _ptr(d_accept_len, torch.int32), _ptr(d_accept_path, torch.int32),
                           _ptr(d_bonus, torch.int32), C.c_void_p(k_pool.data_ptr()), C.c_void_p(v_pool.data_ptr()),
                           _ptr(page_table, torch.int32), C.byref(p), _ptr(d_prefix_len, torch.int32),
                           _ptr(d_tail, torch.int32), _ptr(d_tail_len, torch.int32), _stream())
    _check("war_commit", code)


_lib.war_selftest_bounded_wait.restype = C.c_int
_lib.war_selftest_bounded_wait.argtypes = [C.c_int32, C.c_void_p, C.c_void_p]


def war_selftest_bounded_wait(budget_us: int, d_result: torch.Tensor) -> None:
    """d_result: int64 [4] CUDA tensor; see include/war.h."""
    _check("war_selftest_bounded_wait", _lib.war_selftest_bounded_wait(int(budget_us), _ptr(d_result, torch.int64), _stream()))


def war_device_status() -> int:
    v = C.c_int32(0)
    _check("war_device_status", _lib.war_device_status(_stream(), C.byref(v)))
    return int(v.value)


def new_workspace(params: AttnParams, device) -> torch.Tensor:
    """A device buffer of the size war_verify_attn asks for (torch's allocator returns 512-byte aligned blocks)."""
    n = war_verify_attn_workspace_bytes(params)
    if n == 0:
        raise WarError("war_verify_attn_workspace_bytes", 6)
    return torch.empty(n, dtype=torch.uint8, device=device)


# ---------------------------------------------------------------------------------------------------------------
# rotary store, 8-bit cache, target choice
# ---------------------------------------------------------------------------------------------------------------
KV_TYPES = {torch.bfloat16: 0, torch.float8_e4m3fn: 1, torch.float8_e5m2: 2}
ROPE_KINDS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}


class RopeStoreParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("page_size", C.c_int32), ("max_pages_per_req", C.c_int32), ("kv_type", C.c_int32), ("scale_block", C.c_int32),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_float), ("num_pages", C.c_int64),
                ("q_strides", C.c_int64 * 4), ("k_strides", C.c_int64 * 4), ("v_strides", C.c_int64 * 4),
                ("kpool_strides", C.c_int64 * 4), ("vpool_strides", C.c_int64 * 4)]


class RopeFreqParams(C.Structure):
    _fields_ = [("kind", C.c_int32), ("rot_dim", C.c_int32), ("base", C.c_double), ("scale", C.c_double),
                ("original_length", C.c_double), ("fast", C.c_double), ("slow", C.c_double)]


class AttnQuantParams(C.Structure):
    _fields_ = [("attn", AttnParams), ("kv_type", C.c_int32), ("scale_block", C.c_int32)]


class TargetInputs(C.Structure):
    _fields_ = [("d_ctx", C.c_void_p), ("d_ctx_off", C.c_void_p), ("d_prompt_len", C.c_void_p), ("d_repetition", C.c_void_p),
                ("d_presence", C.c_void_p), ("d_frequency", C.c_void_p), ("d_bias_off", C.c_void_p), ("d_bias_ids", C.c_void_p),
                ("d_bias_val", C.c_void_p), ("d_mask", C.c_void_p)]


class TargetParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("V", C.c_int32), ("dtype", C.c_int32), ("logits_strides", C.c_int64 * 2),
                ("out_strides", C.c_int64 * 2), ("mask_strides", C.c_int64 * 2)]


class CommitQuantParams(C.Structure):
    _fields_ = [("commit", CommitParams), ("kv_type", C.c_int32), ("scale_block", C.c_int32)]


_lib.war_rope_store.restype = C.c_int
_lib.war_rope_store.argtypes = [C.c_void_p] * 8 + [C.POINTER(RopeStoreParams)] + [C.c_void_p] * 6
_lib.war_rope_frequencies.restype = C.c_int
_lib.war_rope_frequencies.argtypes = [C.POINTER(RopeFreqParams), C.c_void_p, C.c_void_p]
_lib.war_verify_attn_quant_workspace_bytes.restype = C.c_size_t
_lib.war_verify_attn_quant_workspace_bytes.argtypes = [C.POINTER(AttnQuantParams)]
_lib.war_verify_attn_quant.restype = C.c_int
_lib.war_verify_attn_quant.argtypes = [C.c_void_p] * 9 + [C.POINTER(AttnQuantParams)] + [C.c_void_p] * 4
_lib.war_target.restype = C.c_int
_lib.war_target.argtypes = [C.c_void_p] * 4 + [C.POINTER(TargetInputs), C.POINTER(TargetParams)] + [C.c_void_p] * 3
_lib.war_commit_quant.restype = C.c_int
_lib.war_commit_quant.argtypes = [C.c_void_p] * 9 + [C.POINTER(CommitQuantParams)] + [C.c_void_p] * 4


def _strided(t: torch.Tensor, ndim: int, *dtypes) -> int:
    """Address of a device tensor that is passed with its strides."""
    if not t.is_cuda or t.dim() != ndim:
        raise ValueError(f"expected a {ndim}-dimensional CUDA tensor")
    if t.dtype not in dtypes:
        raise ValueError(f"expected {' or '.join(map(str, dtypes))}, got {t.dtype}")
    return t.data_ptr()


# What a call works out from its tensors' types, shapes and strides alone is kept by them: for a decoding step's small
# tensors, filling these structures anew takes longer than the kernels.
_by_layout = functools.lru_cache(maxsize=512)


def _layout(t: Optional[torch.Tensor]):
    return None if t is None else (t.dtype, t.shape, t.stride())


def _address(t: Optional[torch.Tensor]) -> Optional[int]:
    """Address of a device tensor whose type and strides have been looked at through _layout."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device buffers must be CUDA tensors")
    return t.data_ptr()


def _stream_of(*tensors: Optional[torch.Tensor]) -> int:
    """The current stream, for a call whose tensors are all on its device."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"the call runs on the current device, cuda:{device}, but a tensor is on cuda:{t.get_device()}")
    return _stream()


def _is_contiguous(t) -> bool:
    """As Tensor.is_contiguous, of a _layout."""
    step = 1
    for size, stride in zip(reversed(t[1]), reversed(t[2])):
        if size != 1 and stride != step and 0 not in t[1]:
            return False
        step *= size
    return True


@_by_layout
def _pool_layout(k_pool, v_pool, k_scale, v_scale):
    """(kv_type, scale_block) of a cache, from _layout of its tensors; checks that pools and scales belong together."""
    kv = KV_TYPES.get(k_pool[0])
    if kv is None or v_pool[0] != k_pool[0] or v_pool[1] != k_pool[1] or len(k_pool[1]) != 4:
        raise ValueError("pools must be [pages, Hkv, page_size, D] of one shape and one of the types " + ", ".join(map(str, KV_TYPES)))
    if kv == 0:
        if k_scale is not None or v_scale is not None:
            raise ValueError("a bf16 cache has no scales")
        return kv, 0
    pages, Hkv, pg, _ = k_pool[1]
    for t in (k_scale, v_scale):
        if t is None or len(t[1]) != 3 or tuple(t[1][:2]) != (pages, Hkv) or t[1][2] < 1 or pg % t[1][2] or t[1] != k_scale[1]:
            raise ValueError("scales must be float32 [pages, Hkv, page_size / scale_block], the same for K and V")
        if t[0] != torch.float32 or not _is_contiguous(t):
            raise ValueError("scales must be contiguous float32")
    return kv, pg // k_scale[1][2]


def _pool_args(k_pool: torch.Tensor, v_pool: torch.Tensor, k_scale, v_scale):
    return _pool_layout(_layout(k_pool), _layout(v_pool), _layout(k_scale), _layout(v_scale))


def _want(t, *want) -> None:
    """Checks the shape in a _layout."""
    if t is not None and tuple(t[1]) != want:
        raise ValueError(f"expected shape {want}, got {tuple(t[1])}")


def war_rope_frequencies(rot_dim: int, base: float, kind: str = "plain", scale: float = 1.0, original_length: float = 0.0,
                         fast: float = 32.0, slow: float = 1.0) -> Tuple[torch.Tensor, float]:
    """(inv_freq float32 [rot_dim / 2] on the host, factor) for war_rope_store; kinds: ROPE_KINDS (see include/war.h)."""
    out = torch.zeros(rot_dim // 2, dtype=torch.float32)
    f = C.c_float(1.0)
    p = RopeFreqParams(ROPE_KINDS[kind], rot_dim, base, scale, original_length, fast, slow)
    _check("war_rope_frequencies", _lib.war_rope_frequencies(C.byref(p), out.data_ptr(), C.addressof(f)))
    return out, float(f.value)


@_by_layout
def _store_params(q, k, v, freq, table, prefix, nodes, parent, k_pool, v_pool, k_scale, v_scale, q_out, interleaved, factor) -> RopeStoreParams:
    if len(k[1]) != 4:
        raise ValueError("d_k must be [B, N, Hkv, D]")
    B, N, Hkv, D = k[1]
    kv, block = _pool_layout(k_pool, v_pool, k_scale, v_scale)
    if k[0] != torch.bfloat16 or v[0] != torch.bfloat16 or (q is not None and q[0] != torch.bfloat16):
        raise ValueError("d_q, d_k and d_v must be bfloat16")
    _want(v, B, N, Hkv, D)
    _want(k_pool, k_pool[1][0], Hkv, k_pool[1][2], D)
    if tuple(prefix) != (B,) or tuple(nodes) != (B,) or tuple(parent) != (B, N):
        raise ValueError("d_prefix_len and d_num_nodes must be [B], d_parent [B, N]")
    if len(table) != 2 or table[0] != B or (q is None) != (q_out is None):
        raise ValueError("page_table must be [B, max_pages]; d_q and d_q_out come together")
    p = RopeStoreParams()
    p.B, p.N, p.Hkv, p.D = B, N, Hkv, D
    if q is not None:
        if len(q[1]) != 4 or tuple(q[1]) != (B, N, q[1][2], D) or q_out != q[1]:
            raise ValueError("d_q and d_q_out must be [B, N, Hq, D]")
        p.Hq, p.q_strides[:] = q[1][2], q[2]
    else:
        p.Hq, p.q_strides[3] = 0, 1
    p.page_size, p.max_pages_per_req, p.num_pages = k_pool[1][2], table[1], k_pool[1][0]
    p.kv_type, p.scale_block, p.rot_dim, p.interleaved, p.factor = kv, block, 2 * math.prod(freq), int(interleaved), factor
    p.k_strides[:], p.v_strides[:], p.kpool_strides[:], p.vpool_strides[:] = k[2], v[2], k_pool[2], v_pool[2]
    return p


def war_rope_store(d_q: Optional[torch.Tensor], d_k: torch.Tensor, d_v: torch.Tensor, d_inv_freq: torch.Tensor, page_table: torch.Tensor,
                   d_prefix_len: torch.Tensor, d_num_nodes: torch.Tensor, d_parent: torch.Tensor, k_pool: torch.Tensor,
                   v_pool: torch.Tensor, k_scale: Optional[torch.Tensor], v_scale: Optional[torch.Tensor],
                   d_q_out: Optional[torch.Tensor], interleaved: bool = False, factor: float = 1.0) -> None:
    """Rotates q (to d_q_out) and k at the slots' places in the text and writes k and v behind prefix_len.  d_q, d_k, d_v:
    bf16 [B, N, H, D], any strides the library accepts (the parts of one projection, say); rot_dim = 2 * len(d_inv_freq).
    Pools [pages, Hkv, page_size, D]: bf16 (no scales), or float8_e4m3fn / float8_e5m2 with float32 scales
    [pages, Hkv, page_size / scale_block]; updated in place.  d_q and d_q_out None: nothing but the store."""
    p = _store_params(_layout(d_q), _layout(d_k), _layout(d_v), d_inv_freq.shape, page_table.shape, d_prefix_len.shape, d_num_nodes.shape,
                      d_parent.shape, _layout(k_pool), _layout(v_pool), _layout(k_scale), _layout(v_scale),
                      None if d_q_out is None else d_q_out.shape, bool(interleaved), float(factor))
    code = _lib.war_rope_store(_address(d_q), _address(d_k), _address(d_v), _ptr(d_inv_freq, torch.float32), _ptr(page_table, torch.int32),
                               _ptr(d_prefix_len, torch.int32), _ptr(d_num_nodes, torch.int32), _ptr(d_parent, torch.int32), C.byref(p),
                               _address(k_pool), _address(v_pool), _address(k_scale), _address(v_scale), _ptr(d_q_out, torch.bfloat16),
                               _stream_of(d_q, d_k, d_v, d_inv_freq, page_table, d_prefix_len, d_num_nodes, d_parent, k_pool, v_pool,
                                          k_scale, v_scale, d_q_out))
    _check("war_rope_store", code)


def attn_quant_params(q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                      page_table: torch.Tensor, scale: float, kernel: int = 0) -> AttnQuantParams:
    kv, block = _pool_args(k_pool, v_pool, k_scale, v_scale)
    if kv == 0:
        raise ValueError("pools must hold 8-bit codes; war_verify_attn reads a bf16 cache")
    if q.shape[3] != k_pool.shape[3] or page_table.dim() != 2 or page_table.shape[0] != q.shape[0]:
        raise ValueError("q [B, N, Hq, D], pools [pages, Hkv, page_size, D], page_table [B, max_pages]")
    return AttnQuantParams(attn_params(q, k_pool, v_pool, page_table, scale, kernel), kv, block)


def war_verify_attn_quant_workspace_bytes(params: AttnQuantParams) -> int:
    return int(_lib.war_verify_attn_quant_workspace_bytes(C.byref(params)))


def new_quant_workspace(params: AttnQuantParams, device) -> torch.Tensor:
    """A device buffer of the size war_verify_attn_quant asks for."""
    n = war_verify_attn_quant_workspace_bytes(params)
    if n == 0:
        raise WarError("war_verify_attn_quant_workspace_bytes", 6)
    return torch.empty(n, dtype=torch.uint8, device=device)


@_by_layout
def _attn_quant_call(q, table, prefix, nodes, parent, out, lse, k_pool, v_pool, k_scale, v_scale, scale, kernel) -> Tuple[bytes, int]:
    """What attn_quant_params gives for these tensors, as bytes, and the workspace's size; checks that they belong together."""
    kv, block = _pool_layout(k_pool, v_pool, k_scale, v_scale)
    if len(q) != 4 or len(table) != 2:
        raise ValueError("d_q must be [B, N, Hq, D], d_page_table [B, max_pages]")
    B, N, Hq, D = q
    num_pages, Hkv, pg, pool_D = k_pool[1]
    for shape, want in ((table[:1], (B,)), (prefix, (B,)), (nodes, (B,)), (parent, (B, N)), (out, (B, N, Hq, D)), (lse, (B, N, Hq)), ((D,), (pool_D,))):
        if shape is not None and tuple(shape) != want:
            raise ValueError(f"expected shape {want}, got {tuple(shape)}")
    p = AttnQuantParams()
    a = p.attn
    a.B, a.N, a.Hq, a.Hkv, a.D, a.page_size, a.max_pages_per_req, a.kernel, a.num_pages, a.scale = B, N, Hq, Hkv, D, pg, table[1], kernel, num_pages, scale
    a.k_strides[:], a.v_strides[:] = k_pool[2], v_pool[2]
    p.kv_type, p.scale_block = kv, block
    return bytes(p), war_verify_attn_quant_workspace_bytes(p)


def war_verify_attn_quant(d_q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                          d_page_table: torch.Tensor, d_prefix_len: torch.Tensor, d_num_nodes: torch.Tensor, d_parent: torch.Tensor,
                          params: AttnQuantParams, d_workspace: torch.Tensor, d_out: torch.Tensor, d_lse: Optional[torch.Tensor]) -> None:
    """war_verify_attn over a float8_e4m3fn / float8_e5m2 cache; params from attn_quant_params for these tensors."""
    a = params.attn
    described, workspace = _attn_quant_call(d_q.shape, d_page_table.shape, d_prefix_len.shape, d_num_nodes.shape, d_parent.shape, d_out.shape,
                                            None if d_lse is None else d_lse.shape, _layout(k_pool), _layout(v_pool), _layout(k_scale),
                                            _layout(v_scale), a.scale, a.kernel)
    if described != bytes(params):
        raise ValueError("params do not describe these tensors (see attn_quant_params)")
    if d_workspace.numel() * d_workspace.element_size() < workspace:
        raise ValueError("workspace is smaller than war_verify_attn_quant_workspace_bytes")
    code = _lib.war_verify_attn_quant(_ptr(d_q, torch.bfloat16), _strided(k_pool, 4, torch.float8_e4m3fn, torch.float8_e5m2),
                                      _strided(v_pool, 4, torch.float8_e4m3fn, torch.float8_e5m2), _ptr(k_scale, torch.float32),
                                      _ptr(v_scale, torch.float32), _ptr(d_page_table, torch.int32), _ptr(d_prefix_len, torch.int32),
                                      _ptr(d_num_nodes, torch.int32), _ptr(d_parent, torch.int32), C.byref(params), _ptr(d_workspace),
                                      _ptr(d_out, torch.bfloat16), _ptr(d_lse, torch.float32),
                                      _stream_of(d_q, k_pool, v_pool, k_scale, v_scale, d_page_table, d_prefix_len, d_num_nodes, d_parent,
                                                 d_workspace, d_out, d_lse))
    _check("war_verify_attn_quant", code)


@_by_layout
def _target_params(logits, out, mask, target, per_slot, per_request, offsets) -> TargetParams:
    if len(logits[1]) != 3:
        raise ValueError("d_logits must be [B, N, V]")
    B, N, V = logits[1]
    p = TargetParams()
    p.B, p.N, p.V, p.dtype = B, N, V, int(logits[0] == torch.float32)
    for t, strides, last in ((logits, p.logits_strides, V), (out, p.out_strides, V), (mask, p.mask_strides, (V + 31) // 32)):
        if t is None:
            continue
        _want(t, B, N, last)
        if t[2][2] != 1 and last > 1:
            raise ValueError("logits, mask and out need unit stride along their last dimension")
        strides[0], strides[1] = t[2][0], t[2][1]
    if out is not None and out[0] != logits[0]:
        raise ValueError("d_out must have the logits' type")
    for shapes, want in (((target,) + per_slot, (B, N)), (per_request, (B,)), (offsets, (B + 1,))):
        for shape in shapes:
            if shape is not None and tuple(shape) != want:
                raise ValueError(f"expected shape {want}, got {tuple(shape)}")
    return p


def war_target(d_logits: torch.Tensor, d_num_nodes: torch.Tensor, d_ids: Optional[torch.Tensor], d_parent: Optional[torch.Tensor],
               d_target: torch.Tensor, d_ctx: Optional[torch.Tensor] = None, d_ctx_off: Optional[torch.Tensor] = None,
               d_prompt_len: Optional[torch.Tensor] = None, d_repetition: Optional[torch.Tensor] = None,
               d_presence: Optional[torch.Tensor] = None, d_frequency: Optional[torch.Tensor] = None,
               d_bias_off: Optional[torch.Tensor] = None, d_bias_ids: Optional[torch.Tensor] = None,
               d_bias_val: Optional[torch.Tensor] = None, d_mask: Optional[torch.Tensor] = None,
               d_out: Optional[torch.Tensor] = None) -> None:
    """Penalties, biases and grammar masks on d_logits (bf16 or float32 [B, N, V], unit stride along V), the chosen token of
    every slot into d_target [B, N] (what war_accept takes), the processed logits into d_out where it is given.
    d_mask: int32 words [B, N, ceil(V / 32)], unit stride along the words; expand() shares one mask."""
    f32, i32, i64 = torch.float32, torch.int32, torch.int64
    if d_ctx is None and not (d_repetition is None and d_presence is None and d_frequency is None):
        raise ValueError("penalties need d_ctx (an empty tensor where all contexts are empty)")
    if d_bias_ids is not None and d_bias_val is not None and d_bias_ids.shape != d_bias_val.shape:
        raise ValueError("d_bias_ids and d_bias_val must be of one length")
    p = _target_params(_layout(d_logits), _layout(d_out), None if d_mask is None else (None, d_mask.shape, d_mask.stride()), d_target.shape,
                       tuple(None if t is None else t.shape for t in (d_ids, d_parent)),
                       tuple(None if t is None else t.shape for t in (d_num_nodes, d_prompt_len, d_repetition, d_presence, d_frequency)),
                       tuple(None if t is None else t.shape for t in (d_ctx_off, d_bias_off)))
    inputs = TargetInputs(_ptr(d_ctx, i32), _ptr(d_ctx_off, i64), _ptr(d_prompt_len, i32), _ptr(d_repetition, f32), _ptr(d_presence, f32),
                          _ptr(d_frequency, f32), _ptr(d_bias_off, i64), _ptr(d_bias_ids, i32), _ptr(d_bias_val, f32),
                          None if d_mask is None else _strided(d_mask, 3, i32))
    if d_bias_off is not None and d_bias_ids is not None and d_bias_val is not None and d_bias_ids.numel() == 0:
        inputs.d_bias_off = inputs.d_bias_ids = inputs.d_bias_val = None             # (an empty tensor has no address)
    code = _lib.war_target(_strided(d_logits, 3, torch.bfloat16, f32), _ptr(d_num_nodes, i32), _ptr(d_ids, i32), _ptr(d_parent, i32),
                           C.byref(inputs), C.byref(p), _ptr(d_target, i32),
                           None if d_out is None else _strided(d_out, 3, torch.bfloat16, f32),
                           _stream_of(d_logits, d_num_nodes, d_ids, d_parent, d_target, d_ctx, d_ctx_off, d_prompt_len, d_repetition,
                                      d_presence, d_frequency, d_bias_off, d_bias_ids, d_bias_val, d_mask, d_out))
    _check("war_target", code)


@_by_layout
def _commit_params(ids, per_slot, per_request, tail, table, k_pool, v_pool, k_scale, v_scale) -> CommitQuantParams:
    if len(ids) != 2 or len(tail) != 2 or len(table) != 2:
        raise ValueError("d_ids must be [B, N], d_tail [B, P], page_table [B, max_pages]")
    q = CommitQuantParams()
    q.kv_type, q.scale_block = _pool_layout(k_pool, v_pool, k_scale, v_scale)
    p = q.commit
    p.B, p.N = ids
    p.P = tail[1]
    for shape, want in ((per_slot, (p.B, p.N)), (tail[:1], (p.B,)), (table[:1], (p.B,))) + tuple((x, (p.B,)) for x in per_request):
        if tuple(shape) != want:
            raise ValueError(f"expected shape {want}, got {tuple(shape)}")
    p.num_pages, p.Hkv, p.page_size, p.D = k_pool[1]
    p.max_pages_per_req = table[1]
    p.k_strides[:], p.v_strides[:] = k_pool[2], v_pool[2]
    return q


def war_commit_quant(d_ids: torch.Tensor, d_accept_len: torch.Tensor, d_accept_path: torch.Tensor, d_bonus: torch.Tensor,
                     k_pool: torch.Tensor, v_pool: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, page_table: torch.Tensor,
                     d_prefix_len: torch.Tensor, d_tail: torch.Tensor, d_tail_len: torch.Tensor) -> None:
    """war_commit for a float8_e4m3fn / float8_e5m2 cache; pools and scales are updated in place.  d_ids and d_accept_path [B, N],
    d_accept_len, d_bonus, d_prefix_len and d_tail_len [B], d_tail [B, P], page_table [B, max_pages]."""
    q = _commit_params(d_ids.shape, d_accept_path.shape, (d_accept_len.shape, d_bonus.shape, d_prefix_len.shape, d_tail_len.shape), d_tail.shape,
                       page_table.shape, _layout(k_pool), _layout(v_pool), _layout(k_scale), _layout(v_scale))
    code = _lib.war_commit_quant(_ptr(d_ids, torch.int32), _ptr(d_accept_len, torch.int32), _ptr(d_accept_path, torch.int32),
                                 _ptr(d_bonus, torch.int32), _address(k_pool), _address(v_pool), _address(k_scale), _address(v_scale),
                                 _ptr(page_table, torch.int32), C.byref(q),
                                 _ptr(d_prefix_len, torch.int32), _ptr(d_tail, torch.int32), _ptr(d_tail_len, torch.int32),
                                 _stream_of(d_ids, d_accept_len, d_accept_path, d_bonus, k_pool, v_pool, k_scale, v_scale, page_table,
                                            d_prefix_len, d_tail, d_tail_len))
    _check("war_commit_quant", code)


# ---------------------------------------------------------------------------------------------------------------
# pages and shared prefixes
# ---------------------------------------------------------------------------------------------------------------
class Pages(NamedTuple):
    """The books of a paged cache, int32 CUDA tensors (see include/war.h): refs [num_pages], free [ceil(num_pages / 32)] (bits),
    page_table [B, max_pages], held [B].  new_pages makes those of an empty pool."""
    refs: torch.Tensor
    free: torch.Tensor
    page_table: torch.Tensor
    held: torch.Tensor


class PagesBooks(C.Structure):
    _fields_ = [("d_refs", C.c_void_p), ("d_free", C.c_void_p), ("d_page_table", C.c_void_p), ("d_held", C.c_void_p), ("B", C.c_int32),
                ("page_size", C.c_int32), ("max_pages_per_req", C.c_int32), ("reserved", C.c_int32), ("num_pages", C.c_int64)]


class PagesCopyParams(C.Structure):
    _fields_ = [("Hkv", C.c_int32), ("D", C.c_int32), ("page_size", C.c_int32), ("kv_type", C.c_int32), ("scale_block", C.c_int32),
                ("reserved", C.c_int32), ("num_pages", C.c_int64), ("kpool_strides", C.c_int64 * 4), ("vpool_strides", C.c_int64 * 4)]


_lib.war_pages_grow.restype = C.c_int
_lib.war_pages_grow.argtypes = [C.POINTER(PagesBooks), C.c_int32] + [C.c_void_p] * 4
_lib.war_pages_fork.restype = C.c_int
_lib.war_pages_fork.argtypes = [C.POINTER(PagesBooks), C.c_void_p, C.c_int32] + [C.c_void_p] * 7
_lib.war_pages_free.restype = C.c_int
_lib.war_pages_free.argtypes = [C.POINTER(PagesBooks)] + [C.c_void_p] * 3
_lib.war_pages_compact_workspace_bytes.restype = C.c_size_t
_lib.war_pages_compact_workspace_bytes.argtypes = [C.c_int64]
_lib.war_pages_compact.restype = C.c_int
_lib.war_pages_compact.argtypes = [C.POINTER(PagesBooks), C.c_void_p, C.c_int32] + [C.c_void_p] * 4
_lib.war_pages_copy.restype = C.c_int
_lib.war_pages_copy.argtypes = [C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p] * 4 + [C.POINTER(PagesCopyParams), C.c_void_p]
_lib.war_prefix_groups.restype = C.c_int
_lib.war_prefix_groups.argtypes = [C.c_void_p] * 3 + [C.c_int32] * 4 + [C.c_void_p] * 3
_lib.war_verify_attn_shared_workspace_bytes.restype = C.c_size_t
_lib.war_verify_attn_shared_workspace_bytes.argtypes = [C.POINTER(AttnParams)]
_lib.war_verify_attn_shared.restype = C.c_int
_lib.war_verify_attn_shared.argtypes = [C.c_void_p] * 9 + [C.POINTER(AttnParams)] + [C.c_void_p] * 4
_lib.war_verify_attn_shared_quant_workspace_bytes.restype = C.c_size_t
_lib.war_verify_attn_shared_quant_workspace_bytes.argtypes = [C.POINTER(AttnQuantParams)]
_lib.war_verify_attn_shared_quant.restype = C.c_int
_lib.war_verify_attn_shared_quant.argtypes = [C.c_void_p] * 11 + [C.POINTER(AttnQuantParams)] + [C.c_void_p] * 4


def new_pages(num_pages: int, B: int, max_pages: int, device) -> Pages:
    """The books of an empty pool for B requests of at most max_pages pages."""
    free = np.zeros(-(-num_pages // 32) * 32, np.uint8)
    free[:num_pages] = 1
    words = torch.from_numpy(np.packbits(free, bitorder="little").view(np.int32))
    zeros = functools.partial(torch.zeros, dtype=torch.int32, device=device)
    return Pages(zeros(num_pages), words.to(device), torch.full((B, max_pages), -1, dtype=torch.int32, device=device), zeros(B))


def _addresses(dtype, first: torch.Tensor, *others: Optional[torch.Tensor]) -> Tuple[list, int]:
    """Addresses of contiguous tensors of one type (None stays None), all on the current device, and its current stream: what _ptr and
    _stream_of look at, in one pass (a call of a few microseconds is bound by this)."""
    device, at = first.get_device(), []
    for t in (first, *others):
        if t is None:
            at.append(None)
        elif t.get_device() == device >= 0 and t.dtype is dtype and t.is_contiguous():
            at.append(t.data_ptr())
        else:
            _ptr(t, dtype)
            break
    else:
        current = torch.cuda.current_device()
        if device == current and _raw_stream is not None:
            return at, _raw_stream(current)
    return at, _stream_of(first, *others)


def _books(pages: Pages, page_size: int, *tensors: Optional[torch.Tensor]) -> Tuple[PagesBooks, list, int]:
    """The structure, the addresses of the call's other tensors, and the stream."""
    refs, free, table, held = pages
    n, width = refs.shape, table.shape
    if len(n) != 1 or len(width) != 2 or held.shape != width[:1] or free.shape != (-(-n[0] // 32),):
        raise ValueError("pages must be refs [num_pages], free [ceil(num_pages / 32)], page_table [B, max_pages], held [B]")
    at, stream = _addresses(torch.int32, refs, free, table, held, *tensors)
    return PagesBooks(at[0], at[1], at[2], at[3], width[0], page_size, width[1], 0, n[0]), at[4:], stream


def _same_shape(want, *tensors) -> None:
    for t in tensors:
        if t is not None and t.shape != want:
            raise ValueError(f"expected shape {tuple(want)}, got {tuple(t.shape)}")


def _copy_list(d_copies: torch.Tensor, least: int) -> int:
    shape = d_copies.shape
    if len(shape) != 2 or shape[1] != 3 or shape[0] < least:
        raise ValueError(f"d_copies must be int32 [n, 3] with n >= {least}")
    return shape[0]


def war_pages_grow(pages: Pages, N: int, page_size: int, d_prefix_len: torch.Tensor, d_tail_len: Optional[torch.Tensor],
                   d_granted: torch.Tensor) -> None:
    """Pages for positions below prefix_len + N of every running request; d_granted [B]: 1 where a request has its room."""
    _same_shape(pages.held.shape, d_prefix_len, d_tail_len, d_granted)
    books, at, stream = _books(pages, page_size, d_prefix_len, d_tail_len, d_granted)
    _check("war_pages_grow", _lib.war_pages_grow(C.byref(books), N, *at, stream))


def war_pages_fork(pages: Pages, d_src: torch.Tensor, page_size: int, d_prefix_len: torch.Tensor, d_tail: torch.Tensor,
                   d_tail_len: torch.Tensor, d_copies: torch.Tensor, d_n_copies: torch.Tensor, d_ok: torch.Tensor) -> None:
    """Request b becomes a copy of request d_src[b] (-1 or b: stays); d_copies int32 [>= B, 3] and d_n_copies [1] for
    war_pages_copy, once per layer; d_ok [1]: 0 where the pool had too few pages and nothing was changed."""
    requests, tail = pages.held.shape, d_tail.shape
    _same_shape(requests, d_src, d_prefix_len, d_tail_len)
    if len(tail) != 2 or tail[:1] != requests or d_n_copies.numel() != 1 or d_ok.numel() != 1:
        raise ValueError("d_tail must be [B, P], d_n_copies and d_ok one number each")
    _copy_list(d_copies, tail[0])
    books, at, stream = _books(pages, page_size, d_src, d_prefix_len, d_tail, d_tail_len, d_copies, d_n_copies, d_ok)
    _check("war_pages_fork", _lib.war_pages_fork(C.byref(books), at[0], tail[1], *at[1:], stream))


def war_pages_free(pages: Pages, d_done: torch.Tensor, d_tail_len: Optional[torch.Tensor] = None) -> None:
    """Requests with d_done[b] != 0 give their pages back and, where d_tail_len is given, stop running (tail_len = -1)."""
    _same_shape(pages.held.shape, d_done, d_tail_len)
    books, at, stream = _books(pages, 1, d_done, d_tail_len)
    _check("war_pages_free", _lib.war_pages_free(C.byref(books), at[0], at[1], stream))


def new_compact_workspace(pages: Pages) -> torch.Tensor:
    n = int(_lib.war_pages_compact_workspace_bytes(pages.refs.numel()))
    if n == 0:
        raise WarError("war_pages_compact_workspace_bytes", 6)
    return torch.empty(n, dtype=torch.uint8, device=pages.refs.device)


def war_pages_compact(pages: Pages, page_size: int, d_workspace: torch.Tensor, d_copies: torch.Tensor, d_n_copies: torch.Tensor,
                      d_top: torch.Tensor) -> None:
    """Moves used pages to the front of the pool, as many as d_copies int32 [n, 3] has lines for; d_n_copies [1], and d_top [1]: no
    page at or above it is in use.  Workspace from new_compact_workspace."""
    if d_workspace.numel() * d_workspace.element_size() < _lib.war_pages_compact_workspace_bytes(pages.refs.numel()):
        raise ValueError("workspace is smaller than war_pages_compact_workspace_bytes")
    if d_n_copies.numel() != 1 or d_top.numel() != 1:
        raise ValueError("d_n_copies and d_top are one number each")
    lines = _copy_list(d_copies, 0)
    books, at, stream = _books(pages, page_size, d_copies, d_n_copies, d_top)
    workspace, _ = _addresses(d_workspace.dtype, d_workspace)
    _check("war_pages_compact", _lib.war_pages_compact(C.byref(books), workspace[0], lines, *at, stream))


@_by_layout
def _copy_params(k_pool, v_pool, k_scale, v_scale) -> PagesCopyParams:
    q = PagesCopyParams()
    q.kv_type, q.scale_block = _pool_layout(k_pool, v_pool, k_scale, v_scale)
    q.num_pages, q.Hkv, q.page_size, q.D = k_pool[1]
    q.kpool_strides[:], q.vpool_strides[:] = k_pool[2], v_pool[2]
    return q


def war_pages_copy(d_copies: torch.Tensor, d_n_copies: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor,
                   k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None) -> None:
    """Applies a list of copies (war_pages_fork, war_pages_compact) to one layer's cache: bf16, or 8-bit with its scales."""
    q = _copy_params(_layout(k_pool), _layout(v_pool), _layout(k_scale), _layout(v_scale))
    lines = _copy_list(d_copies, 0)
    if d_n_copies.numel() != 1:
        raise ValueError("d_n_copies is one number")
    at, _ = _addresses(torch.int32, d_copies, d_n_copies)
    code = _lib.war_pages_copy(at[0], at[1], lines, _address(k_pool), _address(v_pool), _address(k_scale), _address(v_scale), C.byref(q),
                               _stream_of(k_pool, v_pool, k_scale, v_scale))
    _check("war_pages_copy", code)


def war_prefix_groups(d_page_table: torch.Tensor, d_prefix_len: torch.Tensor, d_tail_len: Optional[torch.Tensor], page_size: int,
                      min_shared: int, d_leader: torch.Tensor, d_shared_len: torch.Tensor) -> None:
    """Groups of running requests that share at least min_shared tokens of their prefix: d_leader [B], d_shared_len [B]."""
    shape = d_page_table.shape
    if len(shape) != 2:
        raise ValueError("d_page_table must be [B, max_pages]")
    _same_shape(shape[:1], d_prefix_len, d_tail_len, d_leader, d_shared_len)
    at, stream = _addresses(torch.int32, d_page_table, d_prefix_len, d_tail_len, d_leader, d_shared_len)
    _check("war_prefix_groups", _lib.war_prefix_groups(at[0], at[1], at[2], shape[0], page_size, shape[1], min_shared, at[3], at[4], stream))


def war_verify_attn_shared_workspace_bytes(params: AttnParams) -> int:
    return int(_lib.war_verify_attn_shared_workspace_bytes(C.byref(params)))


def war_verify_attn_shared_quant_workspace_bytes(params: AttnQuantParams) -> int:
    return int(_lib.war_verify_attn_shared_quant_workspace_bytes(C.byref(params)))


def new_shared_workspace(params: AttnParams, device) -> torch.Tensor:
    """A device buffer of the size war_verify_attn_shared asks for."""
    n = war_verify_attn_shared_workspace_bytes(params)
    if n == 0:
        raise WarError("war_verify_attn_shared_workspace_bytes", 6)
    return torch.empty(n, dtype=torch.uint8, device=device)


def new_shared_quant_workspace(params: AttnQuantParams, device) -> torch.Tensor:
    """A device buffer of the size war_verify_attn_shared_quant asks for."""
    n = war_verify_attn_shared_quant_workspace_bytes(params)
    if n == 0:
        raise WarError("war_verify_attn_shared_quant_workspace_bytes", 6)
    return torch.empty(n, dtype=torch.uint8, device=device)


@_by_layout
def _attn_shared_call(q, table, prefix, nodes, parent, leader, shared, out, lse, k_pool, v_pool, k_scale, v_scale, scale, kernel) -> Tuple[bytes, int]:
    """The parameter structure for these tensors, as bytes, and the workspace's size; checks that they belong together."""
    kv, block = _pool_layout(k_pool, v_pool, k_scale, v_scale)
    if len(q) != 4 or len(table) != 2:
        raise ValueError("d_q must be [B, N, Hq, D], d_page_table [B, max_pages]")
    B, N, Hq, D = q
    num_pages, Hkv, pg, pool_D = k_pool[1]
    for shape, want in ((table[:1], (B,)), (prefix, (B,)), (nodes, (B,)), (leader, (B,)), (shared, (B,)), (parent, (B, N)), (out, (B, N, Hq, D)),
                        (lse, (B, N, Hq)), ((D,), (pool_D,))):
        if shape is not None and tuple(shape) != want:
            raise ValueError(f"expected shape {want}, got {tuple(shape)}")
    p = AttnParams() if kv == 0 else AttnQuantParams()
    a = p if kv == 0 else p.attn
    a.B, a.N, a.Hq, a.Hkv, a.D, a.page_size, a.max_pages_per_req, a.kernel, a.num_pages, a.scale = B, N, Hq, Hkv, D, pg, table[1], kernel, num_pages, scale
    a.k_strides[:], a.v_strides[:] = k_pool[2], v_pool[2]
    if kv == 0:
        return bytes(p), war_verify_attn_shared_workspace_bytes(p)
    p.kv_type, p.scale_block = kv, block
    return bytes(p), war_verify_attn_shared_quant_workspace_bytes(p)


def _attn_shared(fn: str, tensors, pools, params, attn: AttnParams, d_workspace, d_out, d_lse) -> None:
    d_q, table, prefix, nodes, parent, leader, shared = tensors
    k_pool, v_pool, k_scale, v_scale = pools
    i32 = torch.int32
    described, workspace = _attn_shared_call(d_q.shape, table.shape, prefix.shape, nodes.shape, parent.shape, leader.shape, shared.shape, d_out.shape,
                                             None if d_lse is None else d_lse.shape, _layout(k_pool), _layout(v_pool), _layout(k_scale),
                                             _layout(v_scale), attn.scale, attn.kernel)
    if described != bytes(params):
        raise ValueError("params do not describe these tensors (see attn_params and attn_quant_params)")
    if d_workspace.numel() * d_workspace.element_size() < workspace:
        raise ValueError(f"workspace is smaller than {fn}_workspace_bytes")
    scales = () if k_scale is None else (_ptr(k_scale, torch.float32), _ptr(v_scale, torch.float32))
    code = getattr(_lib, fn)(_ptr(d_q, torch.bfloat16), _address(k_pool), _address(v_pool), *scales, _ptr(table, i32), _ptr(prefix, i32),
                             _ptr(nodes, i32), _ptr(parent, i32), _ptr(leader, i32), _ptr(shared, i32), C.byref(params), _ptr(d_workspace),
                             _ptr(d_out, torch.bfloat16), _ptr(d_lse, torch.float32), _stream_of(*tensors, *pools, d_workspace, d_out, d_lse))
    _check(fn, code)


def war_verify_attn_shared(d_q: torch.Tensor, d_kpool: torch.Tensor, d_vpool: torch.Tensor, d_page_table: torch.Tensor,
                           d_prefix_len: torch.Tensor, d_num_nodes: torch.Tensor, d_parent: torch.Tensor, d_leader: torch.Tensor,
                           d_shared_len: torch.Tensor, params: AttnParams, d_workspace: torch.Tensor, d_out: torch.Tensor,
                           d_lse: Optional[torch.Tensor]) -> None:
    """war_verify_attn for groups of requests that share a prefix (d_leader, d_shared_len: see war_prefix_groups); params from
    attn_params, workspace from new_shared_workspace."""
    if d_kpool.dtype != torch.bfloat16:
        raise ValueError("pools must be bf16; war_verify_attn_shared_quant reads an 8-bit cache")
    _attn_shared("war_verify_attn_shared", (d_q, d_page_table, d_prefix_len, d_num_nodes, d_parent, d_leader, d_shared_len),
                 (d_kpool, d_vpool, None, None), params, params, d_workspace, d_out, d_lse)


def war_verify_attn_shared_quant(d_q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                                 d_page_table: torch.Tensor, d_prefix_len: torch.Tensor, d_num_nodes: torch.Tensor, d_parent: torch.Tensor,
                                 d_leader: torch.Tensor, d_shared_len: torch.Tensor, params: AttnQuantParams, d_workspace: torch.Tensor,
                                 d_out: torch.Tensor, d_lse: Optional[torch.Tensor]) -> None:
    """war_verify_attn_shared over a float8_e4m3fn / float8_e5m2 cache; params from attn_quant_params, workspace from
    new_shared_quant_workspace."""
    if k_scale is None or v_scale is None:
        raise ValueError("an 8-bit cache has scales; war_verify_attn_shared reads a bf16 cache")
    _attn_shared("war_verify_attn_shared_quant", (d_q, d_page_table, d_prefix_len, d_num_nodes, d_parent, d_leader, d_shared_len),
                 (k_pool, v_pool, k_scale, v_scale), params, params.attn, d_workspace, d_out, d_lse)
