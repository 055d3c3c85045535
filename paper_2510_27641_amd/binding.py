"""Thin ctypes binding of libspecattn.so: argument marshalling only.

Tensors are torch tensors on the GPU (torch is used for device memory and
streams, nothing else); every step of the path runs inside the library's
kernels.  There is no CPU fallback: a missing library is an error.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspecattn.so")

OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE, EUNSUPPORTED, EHIP = 0, -1, -2, -3, -4, -5, -6
ROW_INVALID, ROW_NEAR_BOUNDARY, ROW_OVERFLOW = 1, 2, 4
SEL_BLOCK = 1024
F32, BF16, F16 = 0, 1, 2

EXPORTS = ("specattn_topp_select", "specattn_topp_select_union", "specattn_union_workspace_size", "specattn_sparse_decode_attn", "specattn_sparse_decode_attn_static", "specattn_fused",
           "specattn_workspace_size", "specattn_layer_similarity", "specattn_layer_similarity_workspace_size",
           "specattn_layer_map", "specattn_layer_map_workspace_size", "specattn_check_lists", "specattn_lists_to_csr", "specattn_stream_read",
           "specattn_mx_store", "specattn_mx_load", "specattn_mx_decode_attn", "specattn_mx_workspace_size", "specattn_evict_select", "specattn_evict_workspace_size",
           "specattn_evict_move", "specattn_pages_update", "specattn_pages_workspace_size", "specattn_cache_store", "specattn_prompt_attn",
           "specattn_prompt_workspace_size", "specattn_tree_attn", "specattn_tree_workspace_size", "specattn_init", "specattn_last_error", "specattn_version")


class SelectArgs(C.Structure):
    _fields_ = [
        ("probs", C.c_void_p), ("probs_stride_b", C.c_int64), ("probs_stride_h", C.c_int64),
        ("B", C.c_int32), ("H_kv", C.c_int32), ("n_max", C.c_int32),
        ("seq_lens", C.c_void_p), ("top_p", C.c_float),
        ("indices", C.c_void_p), ("idx_stride_row", C.c_int64), ("idx_capacity", C.c_int32),
        ("counts", C.c_void_p), ("thresholds", C.c_void_p), ("row_flags", C.c_void_p),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32),
        ("emit_physical", C.c_int32),
        ("block_counts", C.c_void_p), ("reuse_selection", C.c_int32),
        ("chunk_size", C.c_int32), ("bisect_iters", C.c_int32),
        ("kept_mask", C.c_void_p),
    ]


class AttnArgs(C.Structure):
    _fields_ = [
        ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("dtype", C.c_int),
        ("B", C.c_int32), ("H_q", C.c_int32), ("H_kv", C.c_int32), ("T", C.c_int32),
        ("d", C.c_int32), ("n_max", C.c_int32), ("sm_scale", C.c_float),
        ("q_stride_b", C.c_int64), ("q_stride_h", C.c_int64), ("q_stride_t", C.c_int64),
        ("kv_stride_b", C.c_int64), ("kv_stride_h", C.c_int64), ("kv_stride_n", C.c_int64),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32),
        ("kv_stride_page", C.c_int64),
        ("seq_lens", C.c_void_p),
        ("indices", C.c_void_p), ("idx_stride_row", C.c_int64), ("counts", C.c_void_p),
        ("idx_capacity", C.c_int32), ("indices_are_physical", C.c_int32),
        ("out", C.c_void_p), ("lse", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
        ("k_new", C.c_void_p), ("v_new", C.c_void_p),
        ("chunk_size", C.c_int32),
        ("out_lowp", C.c_void_p),
    ]


class UnionArgs(C.Structure):
    _fields_ = [
        ("probs", C.c_void_p), ("probs_stride_b", C.c_int64), ("probs_stride_row", C.c_int64),
        ("B", C.c_int32), ("H_draft", C.c_int32), ("S", C.c_int32), ("H_kv", C.c_int32), ("n_max", C.c_int32),
        ("seq_lens", C.c_void_p), ("top_p", C.c_float),
        ("indices", C.c_void_p), ("idx_stride_row", C.c_int64), ("idx_capacity", C.c_int32),
        ("counts", C.c_void_p), ("row_flags", C.c_void_p),
        ("member_thresholds", C.c_void_p), ("member_counts", C.c_void_p),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32),
        ("emit_physical", C.c_int32),
    ]


class MxCache(C.Structure):
    _fields_ = [
        ("codes", C.c_void_p), ("scales", C.c_void_p),
        ("codes_stride_b", C.c_int64), ("codes_stride_h", C.c_int64), ("codes_stride_n", C.c_int64), ("codes_stride_page", C.c_int64),
        ("scales_stride_b", C.c_int64), ("scales_stride_h", C.c_int64), ("scales_stride_n", C.c_int64), ("scales_stride_page", C.c_int64),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32), ("num_pages", C.c_int32),
        ("B", C.c_int32), ("H_kv", C.c_int32), ("n_max", C.c_int32), ("d", C.c_int32),
    ]


class MxRowsArgs(C.Structure):
    _fields_ = [
        ("cache", MxCache), ("k", C.c_void_p), ("v", C.c_void_p), ("dtype", C.c_int), ("T", C.c_int32),
        ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_t", C.c_int64),
        ("starts", C.c_void_p), ("counts", C.c_void_p),
    ]


class MxAttnArgs(C.Structure):
    _fields_ = [
        ("cache", MxCache), ("q", C.c_void_p), ("dtype", C.c_int), ("H_q", C.c_int32), ("T", C.c_int32), ("sm_scale", C.c_float),
        ("q_stride_b", C.c_int64), ("q_stride_h", C.c_int64), ("q_stride_t", C.c_int64),
        ("seq_lens", C.c_void_p), ("indices", C.c_void_p), ("idx_stride_row", C.c_int64), ("counts", C.c_void_p),
        ("idx_capacity", C.c_int32), ("chunk_size", C.c_int32), ("indices_are_physical", C.c_int32),
        ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("out", C.c_void_p), ("out_lowp", C.c_void_p), ("lse", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class EvictArgs(C.Structure):
    _fields_ = [
        ("probs", C.c_void_p), ("probs_stride_b", C.c_int64), ("probs_stride_row", C.c_int64),
        ("B", C.c_int32), ("H", C.c_int32), ("n_max", C.c_int32), ("H_draft", C.c_int32), ("S", C.c_int32),
        ("scores", C.c_void_p), ("positions", C.c_void_p), ("scores_out", C.c_void_p), ("positions_out", C.c_void_p),
        ("row_stride_b", C.c_int64), ("row_stride_h", C.c_int64),
        ("seq_lens", C.c_void_p), ("next_positions", C.c_void_p), ("decay", C.c_double),
        ("budget", C.c_int32), ("sinks", C.c_int32), ("recent", C.c_int32),
        ("move_src", C.c_void_p), ("move_dst", C.c_void_p), ("move_stride_row", C.c_int64), ("move_capacity", C.c_int32),
        ("move_counts", C.c_void_p), ("new_lens", C.c_void_p), ("row_flags", C.c_void_p),
    ]


MAX_PLANES = 8


class MovePlane(C.Structure):
    _fields_ = [
        ("data", C.c_void_p), ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64), ("stride_page", C.c_int64),
        ("row_bytes", C.c_int32), ("H_kv", C.c_int32), ("num_pages", C.c_int32),
    ]


class MoveArgs(C.Structure):
    _fields_ = [
        ("move_src", C.c_void_p), ("move_dst", C.c_void_p), ("move_counts", C.c_void_p), ("move_stride_row", C.c_int64),
        ("move_capacity", C.c_int32), ("B", C.c_int32), ("H", C.c_int32), ("n_max", C.c_int32),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32),
        ("num_planes", C.c_int32), ("planes", MovePlane * MAX_PLANES),
    ]


class PagesArgs(C.Structure):
    _fields_ = [
        ("page_table", C.c_void_p), ("B", C.c_int32), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32), ("num_pages", C.c_int32),
        ("free_pages", C.c_void_p), ("free_count", C.c_void_p), ("free_count_out", C.c_void_p),
        ("seq_lens", C.c_void_p), ("new_lens", C.c_void_p), ("lens_out", C.c_void_p), ("token_starts", C.c_void_p),
        ("slots", C.c_void_p), ("positions", C.c_void_p), ("owners", C.c_void_p), ("token_capacity", C.c_int32), ("row_flags", C.c_void_p),
    ]


class StoreArgs(C.Structure):
    _fields_ = [
        ("k", C.c_void_p), ("v", C.c_void_p), ("dtype", C.c_int), ("B", C.c_int32), ("T", C.c_int32), ("H_kv", C.c_int32), ("d", C.c_int32),
        ("stride_b", C.c_int64), ("stride_t", C.c_int64), ("stride_h", C.c_int64), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
        ("cache_stride_page", C.c_int64), ("cache_stride_h", C.c_int64), ("cache_stride_n", C.c_int64),
        ("num_pages", C.c_int32), ("page_size", C.c_int32), ("slots", C.c_void_p), ("rows", C.c_void_p), ("num_slots", C.c_int32),
    ]


class PromptArgs(C.Structure):
    _fields_ = [
        ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("dtype", C.c_int),
        ("B", C.c_int32), ("H_q", C.c_int32), ("H_kv", C.c_int32), ("d", C.c_int32), ("total_q", C.c_int32), ("total_kv", C.c_int32),
        ("sm_scale", C.c_float), ("q_stride_t", C.c_int64), ("q_stride_h", C.c_int64),
        ("kv_stride_n", C.c_int64), ("kv_stride_h", C.c_int64), ("kv_stride_page", C.c_int64),
        ("q_starts", C.c_void_p), ("kv_starts", C.c_void_p),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32), ("num_pages", C.c_int32),
        ("seq_lens", C.c_void_p), ("out", C.c_void_p), ("out_lowp", C.c_void_p), ("lse", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


MAX_TREE = 64


class TreeArgs(C.Structure):
    _fields_ = [
        ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("dtype", C.c_int),
        ("B", C.c_int32), ("H_q", C.c_int32), ("H_kv", C.c_int32), ("T", C.c_int32), ("d", C.c_int32), ("n_max", C.c_int32),
        ("sm_scale", C.c_float), ("q_stride_b", C.c_int64), ("q_stride_h", C.c_int64), ("q_stride_t", C.c_int64),
        ("kv_stride_b", C.c_int64), ("kv_stride_h", C.c_int64), ("kv_stride_n", C.c_int64), ("kv_stride_page", C.c_int64),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32), ("num_pages", C.c_int32),
        ("tree_masks", C.c_void_p), ("node_counts", C.c_void_p), ("seq_lens", C.c_void_p),
        ("indices", C.c_void_p), ("idx_stride_row", C.c_int64), ("counts", C.c_void_p), ("idx_capacity", C.c_int32),
        ("chunk_size", C.c_int32), ("indices_are_physical", C.c_int32),
        ("out", C.c_void_p), ("out_lowp", C.c_void_p), ("lse", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class SpecAttnError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"specattn status {status}: {text}")
        self.status = status


_lib = None


def load() -> C.CDLL:
    """Load libspecattn.so (built by `python -m paper_2510_27641_amd.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2510_27641_amd.build`")
        lib = C.CDLL(LIB_PATH)
        lib.specattn_topp_select.restype = C.c_int
        lib.specattn_topp_select.argtypes = [C.POINTER(SelectArgs), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.specattn_topp_select_union.restype = C.c_int
        lib.specattn_topp_select_union.argtypes = [C.POINTER(UnionArgs), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.specattn_union_workspace_size.restype = C.c_size_t
        lib.specattn_union_workspace_size.argtypes = [C.POINTER(UnionArgs)]
        lib.specattn_sparse_decode_attn.restype = C.c_int
        lib.specattn_sparse_decode_attn.argtypes = [C.POINTER(AttnArgs), C.c_void_p]
        lib.specattn_sparse_decode_attn_static.restype = C.c_int
        lib.specattn_sparse_decode_attn_static.argtypes = [C.POINTER(AttnArgs), C.c_void_p]
        lib.specattn_fused.restype = C.c_int
        lib.specattn_fused.argtypes = [C.POINTER(SelectArgs), C.POINTER(AttnArgs), C.c_void_p]
        lib.specattn_workspace_size.restype = C.c_size_t
        lib.specattn_workspace_size.argtypes = [C.POINTER(SelectArgs), C.POINTER(AttnArgs)]
        lib.specattn_layer_similarity_workspace_size.restype = C.c_size_t
        lib.specattn_layer_similarity_workspace_size.argtypes = [C.c_int32] * 4
        lib.specattn_layer_similarity.restype = C.c_int
        lib.specattn_layer_similarity.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.specattn_layer_map_workspace_size.restype = C.c_size_t
        lib.specattn_layer_map_workspace_size.argtypes = [C.c_int32] * 2
        lib.specattn_layer_map.restype = C.c_int
        lib.specattn_layer_map.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_size_t, C.c_void_p]
        lib.specattn_check_lists.restype = C.c_int
        lib.specattn_check_lists.argtypes = [C.POINTER(AttnArgs), C.c_int64, C.c_void_p, C.c_void_p]
        lib.specattn_stream_read.restype = C.c_int
        lib.specattn_stream_read.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        lib.specattn_lists_to_csr.restype = C.c_int
        lib.specattn_lists_to_csr.argtypes = [C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        for name, args in (("specattn_mx_store", MxRowsArgs), ("specattn_mx_load", MxRowsArgs), ("specattn_mx_decode_attn", MxAttnArgs),
                           ("specattn_evict_move", MoveArgs), ("specattn_cache_store", StoreArgs), ("specattn_prompt_attn", PromptArgs),
                           ("specattn_tree_attn", TreeArgs)):
            getattr(lib, name).restype = C.c_int
            getattr(lib, name).argtypes = [C.POINTER(args), C.c_void_p]
        lib.specattn_mx_workspace_size.restype = C.c_size_t
        lib.specattn_mx_workspace_size.argtypes = [C.POINTER(MxAttnArgs)]
        for name, args in (("specattn_pages_workspace_size", PagesArgs), ("specattn_prompt_workspace_size", PromptArgs),
                           ("specattn_tree_workspace_size", TreeArgs)):
            getattr(lib, name).restype = C.c_size_t
            getattr(lib, name).argtypes = [C.POINTER(args)]
        lib.specattn_pages_update.restype = C.c_int
        lib.specattn_pages_update.argtypes = [C.POINTER(PagesArgs), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.specattn_evict_select.restype = C.c_int
        lib.specattn_evict_select.argtypes = [C.POINTER(EvictArgs), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.specattn_evict_workspace_size.restype = C.c_size_t
        lib.specattn_evict_workspace_size.argtypes = [C.POINTER(EvictArgs)]
        lib.specattn_init.restype = C.c_int
        lib.specattn_init.argtypes = []
        lib.specattn_last_error.restype = C.c_char_p
        lib.specattn_last_error.argtypes = []
        lib.specattn_version.restype = C.c_int
        lib.specattn_version.argtypes = []
        _lib = lib
    return _lib


def last_error() -> str:
    return load().specattn_last_error().decode()


def _check(status: int):
    if status != OK:
        raise SpecAttnError(status, last_error())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


# The current stream's handle without a Stream object around it: torch.cuda.current_stream() takes 2.7 us, this 0.27, and a selection with
# attention over 8 rows of 1024 positions 13.0 us of host time with one of them per call, more than its kernels.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


# ------------------------------------------------------------------------------------------
# argument structs from tensors
# ------------------------------------------------------------------------------------------
def select_args(probs: torch.Tensor, top_p: float, *, indices: Optional[torch.Tensor],
                counts: torch.Tensor, thresholds: Optional[torch.Tensor] = None,
                row_flags: Optional[torch.Tensor] = None, seq_lens: Optional[torch.Tensor] = None,
                page_table: Optional[torch.Tensor] = None, page_size: int = 0,
                emit_physical: bool = False, block_counts: Optional[torch.Tensor] = None,
                reuse_selection: bool = False, chunk_size: int = 0,
                bisect_iters: int = 0, kept_mask: Optional[torch.Tensor] = None) -> SelectArgs:
    """probs [B,H_kv,n] fp32 (last dim contiguous); indices [B*H_kv, cap] int32."""
    assert probs.dtype == torch.float32 and probs.dim() == 3 and probs.stride(2) == 1
    B, H, n = probs.shape
    a = SelectArgs()
    a.probs = probs.data_ptr()
    a.probs_stride_b, a.probs_stride_h = probs.stride(0), probs.stride(1)
    a.B, a.H_kv, a.n_max = B, H, n
    a.seq_lens = None if seq_lens is None else seq_lens.data_ptr()
    a.top_p = top_p
    if indices is not None:
        assert indices.dtype == torch.int32 and indices.dim() == 2 and indices.stride(1) == 1
        a.indices = indices.data_ptr()
        a.idx_stride_row, a.idx_capacity = indices.stride(0), indices.shape[1]
    a.counts = counts.data_ptr()
    a.thresholds = None if thresholds is None else thresholds.data_ptr()
    a.row_flags = None if row_flags is None else row_flags.data_ptr()
    if page_table is not None:
        assert page_table.dtype == torch.int32 and page_table.is_contiguous()
        a.page_table = page_table.data_ptr()
        a.page_size, a.max_pages_per_seq = page_size, page_table.shape[1]
    a.emit_physical = int(emit_physical)
    if block_counts is not None:
        assert block_counts.dtype == torch.int32 and block_counts.is_contiguous()
        a.block_counts = block_counts.data_ptr()
    a.reuse_selection = int(reuse_selection)
    a.chunk_size = chunk_size
    a.bisect_iters = bisect_iters
    if kept_mask is not None:
        assert kept_mask.dtype == torch.int32 and kept_mask.is_contiguous()
        assert kept_mask.numel() == B * H * ((n + SEL_BLOCK - 1) // SEL_BLOCK) * (SEL_BLOCK // 32)
        a.kept_mask = kept_mask.data_ptr()
    return a


def union_args(probs: torch.Tensor, top_p: float, H_kv: int, *, indices: torch.Tensor, counts: torch.Tensor,
               row_flags: Optional[torch.Tensor] = None, seq_lens: Optional[torch.Tensor] = None,
               member_thresholds: Optional[torch.Tensor] = None, member_counts: Optional[torch.Tensor] = None,
               page_table: Optional[torch.Tensor] = None, page_size: int = 0,
               emit_physical: bool = False) -> UnionArgs:
    """probs [B,H_draft,S,n] fp32 with the (head, step) rows evenly spaced; indices [B*H_kv, cap] int32."""
    assert probs.dtype == torch.float32 and probs.dim() == 4 and probs.stride(3) == 1
    B, H_d, S, n = probs.shape
    assert probs.stride(1) == S * probs.stride(2), "rows (head, step) must be evenly spaced"
    a = UnionArgs()
    a.probs = probs.data_ptr()
    a.probs_stride_b, a.probs_stride_row = probs.stride(0), probs.stride(2)
    a.B, a.H_draft, a.S, a.H_kv, a.n_max = B, H_d, S, H_kv, n
    a.seq_lens = None if seq_lens is None else seq_lens.data_ptr()
    a.top_p = top_p
    assert indices.dtype == torch.int32 and indices.dim() == 2 and indices.stride(1) == 1
    a.indices = indices.data_ptr()
    a.idx_stride_row, a.idx_capacity = indices.stride(0), indices.shape[1]
    a.counts = counts.data_ptr()
    a.row_flags = None if row_flags is None else row_flags.data_ptr()
    a.member_thresholds = None if member_thresholds is None else member_thresholds.data_ptr()
    a.member_counts = None if member_counts is None else member_counts.data_ptr()
    if page_table is not None:
        assert page_table.dtype == torch.int32 and page_table.is_contiguous()
        a.page_table = page_table.data_ptr()
        a.page_size, a.max_pages_per_seq = page_size, page_table.shape[1]
    a.emit_physical = int(emit_physical)
    return a


def attn_args(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, out: torch.Tensor,
              indices: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
              lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
              n_max: Optional[int] = None, sm_scale: float = 0.0,
              page_table: Optional[torch.Tensor] = None, page_size: int = 0,
              indices_are_physical: bool = False, seq_lens: Optional[torch.Tensor] = None,
              k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None,
              chunk_size: int = 0, out_lowp: Optional[torch.Tensor] = None) -> AttnArgs:
    """q [B,H_q,T,d]; contiguous k/v [B,H_kv,n,d]; paged k/v pool [pages,H_kv,page_size,d];
    k_new/v_new [B,H_kv,T,d] contiguous (the new tokens behind the cache), optional."""
    assert q.dim() == 4 and k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride()
    assert q.dtype == k.dtype == v.dtype and q.dtype in (torch.float32, torch.bfloat16, torch.float16)
    assert q.stride(3) == 1 and k.stride(3) == 1
    B, H_q, T, d = q.shape
    paged = page_table is not None or indices_are_physical
    a = AttnArgs()
    a.q, a.k, a.v = q.data_ptr(), k.data_ptr(), v.data_ptr()
    a.dtype = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}[q.dtype]
    a.B, a.H_q, a.H_kv, a.T, a.d = B, H_q, k.shape[1], T, d
    a.sm_scale = sm_scale
    a.q_stride_b, a.q_stride_h, a.q_stride_t = q.stride(0), q.stride(1), q.stride(2)
    if paged:
        a.n_max = int(n_max if n_max is not None else
                      (page_table.shape[1] * page_size if page_table is not None else 0))
        a.kv_stride_page, a.kv_stride_h, a.kv_stride_n = k.stride(0), k.stride(1), k.stride(2)
        a.kv_stride_b = 0
        a.page_size = page_size
        if page_table is not None:
            assert page_table.dtype == torch.int32 and page_table.is_contiguous()
            a.page_table = page_table.data_ptr()
            a.max_pages_per_seq = page_table.shape[1]
    else:
        a.n_max = k.shape[2] if n_max is None else n_max
        a.kv_stride_b, a.kv_stride_h, a.kv_stride_n = k.stride(0), k.stride(1), k.stride(2)
    a.seq_lens = None if seq_lens is None else seq_lens.data_ptr()
    if indices is not None:
        assert indices.dtype == torch.int32 and indices.dim() == 2 and indices.stride(1) == 1
        a.indices = indices.data_ptr()
        a.idx_stride_row, a.idx_capacity = indices.stride(0), indices.shape[1]
    a.counts = None if counts is None else counts.data_ptr()
    a.indices_are_physical = int(indices_are_physical)
    assert out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == (B, H_q, T, d)
    a.out = out.data_ptr()
    a.lse = None if lse is None else lse.data_ptr()
    a.chunk_size = chunk_size
    if out_lowp is not None:
        assert out_lowp.dtype == q.dtype and out_lowp.is_contiguous() and tuple(out_lowp.shape) == (B, H_q, T, d)
        a.out_lowp = out_lowp.data_ptr()
    if k_new is not None:
        assert v_new is not None and k_new.dtype == v_new.dtype == q.dtype
        assert k_new.is_contiguous() and v_new.is_contiguous()
        assert tuple(k_new.shape) == tuple(v_new.shape) == (B, a.H_kv, T, d)
        a.k_new, a.v_new = k_new.data_ptr(), v_new.data_ptr()
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    return a


def mx_cache(codes: torch.Tensor, scales: torch.Tensor, *, page_table: Optional[torch.Tensor] = None, n_max: Optional[int] = None,
             B: Optional[int] = None) -> MxCache:
    """A cache in 4 bits.  Contiguous: codes uint8 [B,H_kv,n,d], scales uint8 [B,H_kv,n,d/16].  Paged: pools
    [pages,H_kv,page_size,d] and [pages,H_kv,page_size,d/16] with page_table [B,max_pages] int32 (a pool without a page table, for
    lists of pool slots: give B).  n_max: slots per sequence, all of them unless given."""
    assert codes.dtype == scales.dtype == torch.uint8 and codes.dim() == scales.dim() == 4
    assert codes.stride(3) == scales.stride(3) == 1 and codes.shape[:3] == scales.shape[:3] and scales.shape[3] * 16 == codes.shape[3]
    c = MxCache()
    c.codes, c.scales = codes.data_ptr(), scales.data_ptr()
    c.H_kv, c.d = codes.shape[1], codes.shape[3]
    c.codes_stride_h, c.codes_stride_n = codes.stride(1), codes.stride(2)
    c.scales_stride_h, c.scales_stride_n = scales.stride(1), scales.stride(2)
    if page_table is None and B is None:
        c.B, c.n_max = codes.shape[0], codes.shape[2] if n_max is None else n_max
        assert c.n_max <= codes.shape[2]
        c.codes_stride_b, c.scales_stride_b = codes.stride(0), scales.stride(0)
        return c
    c.num_pages, c.page_size = codes.shape[0], codes.shape[2]
    c.codes_stride_page, c.scales_stride_page = codes.stride(0), scales.stride(0)
    if page_table is not None:
        assert page_table.dtype == torch.int32 and page_table.is_contiguous()
        c.page_table = page_table.data_ptr()
        c.B, c.max_pages_per_seq = page_table.shape
        c.n_max = c.max_pages_per_seq * c.page_size if n_max is None else n_max
    else:
        c.B, c.n_max = B, c.num_pages * c.page_size if n_max is None else n_max
    return c


_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _int32(t: Optional[torch.Tensor], n: int):
    if t is None:
        return None
    assert t.dtype == torch.int32 and t.is_contiguous() and t.numel() == n
    return t.data_ptr()


def mx_rows_args(cache: MxCache, k: torch.Tensor, v: torch.Tensor, *, starts: Optional[torch.Tensor] = None,
                 counts: Optional[torch.Tensor] = None) -> MxRowsArgs:
    """k, v [B,H_kv,T,d] (last dim contiguous, equal strides): rows for slots starts[b] .. starts[b] + counts[b] - 1."""
    assert k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and k.stride(3) == 1
    assert k.shape[0] == cache.B and k.shape[1] == cache.H_kv and k.shape[3] == cache.d
    a = MxRowsArgs()
    a.cache = cache
    a.k, a.v, a.dtype, a.T = k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], k.shape[2]
    a.stride_b, a.stride_h, a.stride_t = k.stride(0), k.stride(1), k.stride(2)
    a.starts, a.counts = _int32(starts, cache.B), _int32(counts, cache.B)
    return a


def mx_attn_args(q: torch.Tensor, cache: MxCache, *, out: Optional[torch.Tensor] = None, out_lowp: Optional[torch.Tensor] = None,
                 lse: Optional[torch.Tensor] = None, indices: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
                 seq_lens: Optional[torch.Tensor] = None, sm_scale: float = 0.0, chunk_size: int = 0, indices_are_physical: bool = False,
                 k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> MxAttnArgs:
    """q [B,H_q,T,d] bf16 or fp16; the other arguments as for attn_args."""
    assert q.dim() == 4 and q.stride(3) == 1 and q.dtype in _DTYPES and q.shape[0] == cache.B and q.shape[3] == cache.d
    B, H_q, T, d = q.shape
    a = MxAttnArgs()
    a.cache = cache
    a.q, a.dtype, a.H_q, a.T, a.sm_scale = q.data_ptr(), _DTYPES[q.dtype], H_q, T, sm_scale
    a.q_stride_b, a.q_stride_h, a.q_stride_t = q.stride(0), q.stride(1), q.stride(2)
    a.seq_lens = _int32(seq_lens, B)
    if indices is not None:
        assert indices.dtype == torch.int32 and indices.dim() == 2 and indices.stride(1) == 1 and indices.shape[0] == B * cache.H_kv
        a.indices = indices.data_ptr()
        a.idx_stride_row, a.idx_capacity = indices.stride(0), indices.shape[1]
    a.counts = _int32(counts, B * cache.H_kv)
    a.chunk_size, a.indices_are_physical = chunk_size, int(indices_are_physical)
    if out is not None:
        assert out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == (B, H_q, T, d)
        a.out = out.data_ptr()
    if out_lowp is not None:
        assert out_lowp.dtype == q.dtype and out_lowp.is_contiguous() and tuple(out_lowp.shape) == (B, H_q, T, d)
        a.out_lowp = out_lowp.data_ptr()
    if lse is not None:
        assert lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (B, H_q, T)
        a.lse = lse.data_ptr()
    for name, t in (("k_new", k_new), ("v_new", v_new)):
        if t is not None:
            assert t.dtype == q.dtype and t.is_contiguous() and tuple(t.shape) == (B, cache.H_kv, T, d)
            setattr(a, name, t.data_ptr())
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    return a


def evict_args(probs: Optional[torch.Tensor], scores: torch.Tensor, positions: torch.Tensor, next_positions: torch.Tensor, budget: int, *,
               move_src: torch.Tensor, move_dst: torch.Tensor, move_counts: torch.Tensor, new_lens: torch.Tensor,
               scores_out: Optional[torch.Tensor] = None, positions_out: Optional[torch.Tensor] = None,
               seq_lens: Optional[torch.Tensor] = None, sinks: int = 0, recent: int = 0, decay: float = 1.0,
               row_flags: Optional[torch.Tensor] = None) -> EvictArgs:
    """probs [B,H_draft,S,n] fp32 as for union_args, or None; scores [B,H,n] fp32 and positions [B,H,n] int32, updated in place
    unless scores_out and positions_out are given; move_src and move_dst [B*H, cap] int32, cap >= min(budget, n - budget).
    Whoever appends tokens behind new_lens writes their places in the text into positions before the next call."""
    B, H, n = scores.shape
    scores_out, positions_out = scores if scores_out is None else scores_out, positions if positions_out is None else positions_out
    for t, dtype in ((scores, torch.float32), (scores_out, torch.float32), (positions, torch.int32), (positions_out, torch.int32)):
        assert t.dtype == dtype and tuple(t.shape) == (B, H, n) and t.stride() == scores.stride() and t.stride(2) == 1
    a = EvictArgs()
    a.B, a.H, a.n_max = B, H, n
    if probs is not None:
        assert probs.dtype == torch.float32 and probs.dim() == 4 and probs.stride(3) == 1 and probs.shape[0] == B and probs.shape[3] == n
        assert probs.stride(1) == probs.shape[2] * probs.stride(2), "rows (head, step) must be evenly spaced"
        a.probs, a.H_draft, a.S = probs.data_ptr(), probs.shape[1], probs.shape[2]
        a.probs_stride_b, a.probs_stride_row = probs.stride(0), probs.stride(2)
    a.scores, a.positions, a.scores_out, a.positions_out = scores.data_ptr(), positions.data_ptr(), scores_out.data_ptr(), positions_out.data_ptr()
    a.row_stride_b, a.row_stride_h = scores.stride(0), scores.stride(1)
    a.seq_lens, a.next_positions = _int32(seq_lens, B), _int32(next_positions, B)
    a.decay, a.budget, a.sinks, a.recent = decay, budget, sinks, recent
    assert move_src.dtype == move_dst.dtype == torch.int32 and move_src.shape == move_dst.shape and move_src.stride() == move_dst.stride()
    assert move_src.dim() == 2 and move_src.shape[0] == B * H and move_src.stride(1) == 1
    a.move_src, a.move_dst = move_src.data_ptr(), move_dst.data_ptr()
    a.move_stride_row, a.move_capacity = move_src.stride(0), move_src.shape[1]
    a.move_counts, a.new_lens, a.row_flags = _int32(move_counts, B * H), _int32(new_lens, B), _int32(row_flags, B * H)
    return a


def move_args(move_src: torch.Tensor, move_dst: torch.Tensor, move_counts: torch.Tensor, planes, *, B: int,
              page_table: Optional[torch.Tensor] = None, n_max: Optional[int] = None) -> MoveArgs:
    """planes: up to MAX_PLANES tensors [B,H_kv,n,.] or, with page_table [B,max_pages] int32, pools [pages,H_kv,page_size,.], any type.
    Pages that slots are moved to must belong to one sequence alone."""
    assert move_src.dtype == move_dst.dtype == torch.int32 and move_src.shape == move_dst.shape and move_src.stride() == move_dst.stride()
    assert move_src.dim() == 2 and move_src.stride(1) == 1 and move_src.shape[0] % B == 0
    a = MoveArgs()
    a.move_src, a.move_dst, a.move_counts = move_src.data_ptr(), move_dst.data_ptr(), _int32(move_counts, move_src.shape[0])
    a.move_stride_row, a.move_capacity = move_src.stride(0), move_src.shape[1]
    a.B, a.H = B, move_src.shape[0] // B
    assert 1 <= len(planes) <= MAX_PLANES
    slots = planes[0].shape[2]
    if page_table is not None:
        assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.shape[0] == B
        a.page_table, a.page_size, a.max_pages_per_seq = page_table.data_ptr(), slots, page_table.shape[1]
        slots *= page_table.shape[1]
    a.n_max = slots if n_max is None else n_max
    a.num_planes = len(planes)
    for p, t in zip(a.planes, planes):
        size = t.element_size()
        assert t.dim() == 4 and t.stride(3) == 1
        assert t.shape[2] == a.page_size if page_table is not None else t.shape[0] == B and t.shape[2] >= a.n_max
        p.data, p.H_kv, p.row_bytes = t.data_ptr(), t.shape[1], t.shape[3] * size
        p.stride_h, p.stride_n = t.stride(1) * size, t.stride(2) * size
        if page_table is not None:
            p.stride_page, p.num_pages = t.stride(0) * size, t.shape[0]
        else:
            p.stride_b = t.stride(0) * size
    return a


def pages_args(page_table: torch.Tensor, page_size: int, free_pages: torch.Tensor, free_count: torch.Tensor, seq_lens: torch.Tensor,
               new_lens: torch.Tensor, *, lens_out: Optional[torch.Tensor] = None, free_count_out: Optional[torch.Tensor] = None,
               token_starts: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
               owners: Optional[torch.Tensor] = None, row_flags: Optional[torch.Tensor] = None) -> PagesArgs:
    """page_table [B,max_pages], free_pages [pages], free_count [1], seq_lens and new_lens [B], all int32; seq_lens and free_count are
    updated in place unless lens_out and free_count_out are given.  slots (and positions, owners): [capacity] int32."""
    assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.dim() == 2
    B = page_table.shape[0]
    a = PagesArgs()
    a.page_table, a.B, a.max_pages_per_seq = page_table.data_ptr(), B, page_table.shape[1]
    a.page_size, a.num_pages = page_size, free_pages.numel()
    a.free_pages, a.free_count = _int32(free_pages, free_pages.numel()), _int32(free_count, 1)
    a.free_count_out = _int32(free_count if free_count_out is None else free_count_out, 1)
    a.seq_lens, a.new_lens = _int32(seq_lens, B), _int32(new_lens, B)
    a.lens_out = _int32(seq_lens if lens_out is None else lens_out, B)
    a.token_starts, a.row_flags = _int32(token_starts, B + 1), _int32(row_flags, B)
    if slots is not None:
        a.token_capacity = slots.numel()
        a.slots = _int32(slots, slots.numel())
    a.positions, a.owners = _int32(positions, a.token_capacity), _int32(owners, a.token_capacity)
    return a


def store_args(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, slots: torch.Tensor, *,
               rows: Optional[torch.Tensor] = None) -> StoreArgs:
    """k, v: packed rows [N,H_kv,d], or [B,H_kv,T,d], whose row b * T + t is node t of sequence b; caches: pools [pages,H_kv,page_size,d] (or
    contiguous [B,H_kv,n,d], slots b * n + position); slots [M] int32, -1 for none; rows [M] int32: the source row of each slot."""
    assert k.shape == v.shape and k.stride() == v.stride() and k.stride(-1) == 1 and k_cache.shape == v_cache.shape and k_cache.stride() == v_cache.stride()
    assert k.dtype == v.dtype == k_cache.dtype == v_cache.dtype and k.dtype in _DTYPES and k.dim() in (3, 4) and k_cache.dim() == 4 and k_cache.stride(3) == 1
    a = StoreArgs()
    a.k, a.v, a.dtype = k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype]
    if k.dim() == 3:
        a.B, a.T, a.stride_t, a.stride_h = 1, k.shape[0], k.stride(0), k.stride(1)
    else:
        a.B, a.T, a.stride_b, a.stride_t, a.stride_h = k.shape[0], k.shape[2], k.stride(0), k.stride(2), k.stride(1)
    a.H_kv, a.d = k.shape[1], k.shape[-1]
    assert k_cache.shape[1] == a.H_kv and k_cache.shape[3] == a.d
    a.k_cache, a.v_cache = k_cache.data_ptr(), v_cache.data_ptr()
    a.num_pages, a.page_size = k_cache.shape[0], k_cache.shape[2]
    a.cache_stride_page, a.cache_stride_h, a.cache_stride_n = k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)
    a.num_slots = slots.numel()
    a.slots, a.rows = _int32(slots, a.num_slots), _int32(rows, a.num_slots)
    return a


def _outputs(a, shape, dtype, out, out_lowp, lse):
    if out is not None:
        assert out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == shape
        a.out = out.data_ptr()
    if out_lowp is not None:
        assert out_lowp.dtype == dtype and out_lowp.is_contiguous() and tuple(out_lowp.shape) == shape
        a.out_lowp = out_lowp.data_ptr()
    if lse is not None:
        assert lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == shape[:-1]
        a.lse = lse.data_ptr()


def prompt_args(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_starts: torch.Tensor, *, kv_starts: Optional[torch.Tensor] = None,
                page_table: Optional[torch.Tensor] = None, seq_lens: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                out_lowp: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, sm_scale: float = 0.0,
                workspace: Optional[torch.Tensor] = None) -> PromptArgs:
    """q [rows,H_q,d] bf16 or fp16; k, v [kv_rows,H_kv,d] or, with page_table [B,max_pages] and seq_lens [B], pools [pages,H_kv,page_size,d];
    q_starts, kv_starts [B+1] int32; out, out_lowp [rows,H_q,d]; lse [rows,H_q]."""
    assert q.dim() == 3 and k.shape == v.shape and k.stride() == v.stride() and q.dtype == k.dtype == v.dtype and q.dtype in _DTYPES
    assert q.stride(2) == 1 and k.stride(-1) == 1 and k.shape[-1] == q.shape[2] and k.dim() == (3 if page_table is None else 4)
    a = PromptArgs()
    B = q_starts.numel() - 1
    a.q, a.k, a.v, a.dtype = q.data_ptr(), k.data_ptr(), v.data_ptr(), _DTYPES[q.dtype]
    a.B, a.H_q, a.H_kv, a.d, a.total_q, a.sm_scale = B, q.shape[1], k.shape[1], q.shape[2], q.shape[0], sm_scale
    a.q_stride_t, a.q_stride_h, a.kv_stride_h = q.stride(0), q.stride(1), k.stride(1)
    a.q_starts, a.kv_starts = _int32(q_starts, B + 1), _int32(kv_starts, B + 1)
    if page_table is None:
        a.total_kv, a.kv_stride_n = k.shape[0], k.stride(0)
        assert seq_lens is None and (kv_starts is not None or k.shape[0] >= q.shape[0])
    else:
        assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.shape[0] == B
        a.page_table, a.max_pages_per_seq, a.num_pages, a.page_size = page_table.data_ptr(), page_table.shape[1], k.shape[0], k.shape[2]
        a.kv_stride_page, a.kv_stride_n = k.stride(0), k.stride(2)
        a.seq_lens = _int32(seq_lens, B)
    _outputs(a, tuple(q.shape), q.dtype, out, out_lowp, lse)
    if workspace is not None:
        set_workspace(a, workspace)
    return a


def tree_args(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, tree_masks: torch.Tensor, *,
              out: Optional[torch.Tensor] = None, out_lowp: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
              indices: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None, node_counts: Optional[torch.Tensor] = None,
              seq_lens: Optional[torch.Tensor] = None, n_max: Optional[int] = None, sm_scale: float = 0.0, chunk_size: int = 0,
              page_table: Optional[torch.Tensor] = None, page_size: int = 0, indices_are_physical: bool = False,
              workspace: Optional[torch.Tensor] = None) -> TreeArgs:
    """q [B,H_q,T,d] bf16 or fp16; k, v, lists and pages as for attn_args; k_new, v_new [B,H_kv,T,d] contiguous; tree_masks [B,T] int64,
    bit u of word t set where node t attends to node u; node_counts [B] int32."""
    assert q.dim() == 4 and k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and q.dtype == k.dtype == v.dtype and q.dtype in _DTYPES
    assert q.stride(3) == 1 and k.stride(3) == 1 and k.shape[3] == q.shape[3]
    B, H_q, T, d = q.shape
    a = TreeArgs()
    a.q, a.k, a.v, a.dtype = q.data_ptr(), k.data_ptr(), v.data_ptr(), _DTYPES[q.dtype]
    a.B, a.H_q, a.H_kv, a.T, a.d, a.sm_scale = B, H_q, k.shape[1], T, d, sm_scale
    a.q_stride_b, a.q_stride_h, a.q_stride_t = q.stride(0), q.stride(1), q.stride(2)
    a.kv_stride_h, a.kv_stride_n = k.stride(1), k.stride(2)
    for name, t in (("k_new", k_new), ("v_new", v_new)):
        assert t.dtype == q.dtype and t.is_contiguous() and tuple(t.shape) == (B, a.H_kv, T, d)
        setattr(a, name, t.data_ptr())
    assert tree_masks.dtype == torch.int64 and tree_masks.is_contiguous() and tuple(tree_masks.shape) == (B, T)
    a.tree_masks = tree_masks.data_ptr()
    if page_table is not None or indices_are_physical:
        a.kv_stride_page, a.num_pages, a.page_size = k.stride(0), k.shape[0], k.shape[2]
        assert page_size in (0, k.shape[2])
        slots = k.shape[0] * k.shape[2]
        if page_table is not None:
            assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.shape[0] == B
            a.page_table, a.max_pages_per_seq = page_table.data_ptr(), page_table.shape[1]
            slots = page_table.shape[1] * k.shape[2]
        a.n_max = slots if n_max is None else n_max
    else:
        assert k.shape[0] == B
        a.kv_stride_b, a.n_max = k.stride(0), k.shape[2] if n_max is None else n_max
        assert a.n_max <= k.shape[2]
    a.node_counts, a.seq_lens, a.counts = _int32(node_counts, B), _int32(seq_lens, B), _int32(counts, B * a.H_kv)
    if indices is not None:
        assert indices.dtype == torch.int32 and indices.dim() == 2 and indices.stride(1) == 1 and indices.shape[0] == B * a.H_kv
        a.indices, a.idx_stride_row, a.idx_capacity = indices.data_ptr(), indices.stride(0), indices.shape[1]
    a.chunk_size, a.indices_are_physical = chunk_size, int(indices_are_physical)
    _outputs(a, (B, H_q, T, d), q.dtype, out, out_lowp, lse)
    if workspace is not None:
        set_workspace(a, workspace)
    return a


def set_workspace(args, workspace: torch.Tensor) -> None:
    """The workspace of argument structs that carry one."""
    args.workspace, args.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()


# ------------------------------------------------------------------------------------------
# the entry points (same names as the C ABI)
# ------------------------------------------------------------------------------------------
def specattn_workspace_size(sel: Optional[SelectArgs], attn: Optional[AttnArgs]) -> int:
    return int(load().specattn_workspace_size(None if sel is None else C.byref(sel),
                                              None if attn is None else C.byref(attn)))


def specattn_topp_select(sel: SelectArgs, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().specattn_topp_select(C.byref(sel), _ptr(workspace), nbytes, _stream(stream)))


def specattn_union_workspace_size(args: UnionArgs) -> int:
    return int(load().specattn_union_workspace_size(C.byref(args)))


def specattn_topp_select_union(args: UnionArgs, workspace: torch.Tensor, stream=None) -> None:
    nbytes = workspace.numel() * workspace.element_size()
    _check(load().specattn_topp_select_union(C.byref(args), _ptr(workspace), nbytes, _stream(stream)))


def specattn_sparse_decode_attn(attn: AttnArgs, stream=None) -> None:
    _check(load().specattn_sparse_decode_attn(C.byref(attn), _stream(stream)))


def specattn_sparse_decode_attn_static(attn: AttnArgs, stream=None) -> None:
    """The same call on the library's built-in scratch buffer: allocates nothing, ignores attn.workspace."""
    _check(load().specattn_sparse_decode_attn_static(C.byref(attn), _stream(stream)))


def specattn_layer_similarity(attn_draft: torch.Tensor, attn_verifier: torch.Tensor, S: torch.Tensor,
                              workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """attn_draft [m, rows, L], attn_verifier [n, rows, L] fp32 contiguous; S [m, n] fp64 (out)."""
    assert attn_draft.dtype == attn_verifier.dtype == torch.float32 and S.dtype == torch.float64
    assert attn_draft.is_contiguous() and attn_verifier.is_contiguous() and S.is_contiguous()
    m, rows, L = attn_draft.shape
    n = attn_verifier.shape[0]
    assert tuple(attn_verifier.shape[1:]) == (rows, L) and tuple(S.shape) == (m, n)
    ws = workspace if workspace is not None else alloc_workspace(int(load().specattn_layer_similarity_workspace_size(m, n, rows, L)))
    _check(load().specattn_layer_similarity(_ptr(attn_draft), _ptr(attn_verifier), m, n, rows, L, _ptr(S), _ptr(ws),
                                            ws.numel(), _stream(stream)))


def specattn_layer_map(S: torch.Tensor, f: torch.Tensor, total: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                       stream=None) -> None:
    """S [m, n] fp64 contiguous; f [n] int32 (out); total [1] fp64 (out)."""
    assert S.dtype == torch.float64 and S.is_contiguous() and S.dim() == 2
    m, n = S.shape
    assert f.dtype == torch.int32 and f.numel() == n and total.dtype == torch.float64 and total.numel() == 1
    ws = workspace if workspace is not None else alloc_workspace(int(load().specattn_layer_map_workspace_size(m, n)))
    _check(load().specattn_layer_map(_ptr(S), m, n, _ptr(f), _ptr(total), _ptr(ws), ws.numel(), _stream(stream)))


def specattn_fused(sel: SelectArgs, attn: AttnArgs, stream=None) -> None:
    _check(load().specattn_fused(C.byref(sel), C.byref(attn), _stream(stream)))


def specattn_lists_to_csr(indices: Optional[torch.Tensor], counts: torch.Tensor, indptr: torch.Tensor,
                          packed: Optional[torch.Tensor] = None, capacity: Optional[int] = None, stream=None) -> None:
    """indptr [rows + 1] int64 <- exclusive prefix of the list lengths; packed (optional) <- the lists back to back."""
    assert counts.dtype == torch.int32 and indptr.dtype == torch.int64 and indptr.numel() == counts.numel() + 1
    stride = 0 if indices is None else indices.stride(0)
    cap = capacity if capacity is not None else (indices.shape[1] if indices is not None else 2 ** 31 - 1)
    _check(load().specattn_lists_to_csr(_ptr(indices), stride, cap, _ptr(counts), counts.numel(), _ptr(indptr), _ptr(packed),
                                        _stream(stream)))


def specattn_mx_store(args: MxRowsArgs, stream=None) -> None:
    """Rows of keys and values into a 4-bit cache."""
    _check(load().specattn_mx_store(C.byref(args), _stream(stream)))


def specattn_mx_load(args: MxRowsArgs, stream=None) -> None:
    """The values that slots of a 4-bit cache stand for, into args.k and args.v."""
    _check(load().specattn_mx_load(C.byref(args), _stream(stream)))


def specattn_mx_workspace_size(args: MxAttnArgs) -> int:
    return int(load().specattn_mx_workspace_size(C.byref(args)))


def specattn_mx_decode_attn(args: MxAttnArgs, stream=None) -> None:
    _check(load().specattn_mx_decode_attn(C.byref(args), _stream(stream)))


def specattn_evict_workspace_size(args: EvictArgs) -> int:
    return int(load().specattn_evict_workspace_size(C.byref(args)))


def specattn_evict_select(args: EvictArgs, workspace: torch.Tensor, stream=None) -> None:
    nbytes = workspace.numel() * workspace.element_size()
    _check(load().specattn_evict_select(C.byref(args), _ptr(workspace), nbytes, _stream(stream)))


def specattn_evict_move(args: MoveArgs, stream=None) -> None:
    _check(load().specattn_evict_move(C.byref(args), _stream(stream)))


def specattn_pages_workspace_size(args: PagesArgs) -> int:
    return int(load().specattn_pages_workspace_size(C.byref(args)))


def specattn_pages_update(args: PagesArgs, workspace: torch.Tensor, stream=None) -> None:
    """Page tables, free pages and the slots of new tokens, from the lengths that sequences have and are to have."""
    nbytes = workspace.numel() * workspace.element_size()
    _check(load().specattn_pages_update(C.byref(args), _ptr(workspace), nbytes, _stream(stream)))


def specattn_cache_store(args: StoreArgs, stream=None) -> None:
    """Rows of keys and values into the slots of a cache."""
    _check(load().specattn_cache_store(C.byref(args), _stream(stream)))


def specattn_prompt_workspace_size(args: PromptArgs) -> int:
    return int(load().specattn_prompt_workspace_size(C.byref(args)))


def specattn_prompt_attn(args: PromptArgs, stream=None) -> None:
    """Causal attention over packed prompts, alone or behind a prefix in pages."""
    _check(load().specattn_prompt_attn(C.byref(args), _stream(stream)))


def specattn_tree_workspace_size(args: TreeArgs) -> int:
    return int(load().specattn_tree_workspace_size(C.byref(args)))


def specattn_tree_attn(args: TreeArgs, stream=None) -> None:
    """Sparse decode attention of a tree of drafted tokens."""
    _check(load().specattn_tree_attn(C.byref(args), _stream(stream)))


def specattn_init() -> None:
    """One-time set-up of the current device (kernel attributes); needed only before capturing a first call."""
    _check(load().specattn_init())


def specattn_check_lists(attn: AttnArgs, n_bad: torch.Tensor, pool_slots: int = 0, stream=None) -> None:
    """Counts the index-list violations of an attention call into n_bad (int32 device tensor of one element)."""
    assert n_bad.dtype == torch.int32 and n_bad.numel() == 1
    _check(load().specattn_check_lists(C.byref(attn), pool_slots, _ptr(n_bad), _stream(stream)))


def specattn_stream_read(src: torch.Tensor, sink: Optional[torch.Tensor] = None, stream=None) -> None:
    """Plain read of every byte of `src` (contiguous); the caller times it."""
    assert src.is_contiguous()
    _check(load().specattn_stream_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream(stream)))


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A 256-byte aligned device buffer of at least nbytes (torch's allocator aligns to 512)."""
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
