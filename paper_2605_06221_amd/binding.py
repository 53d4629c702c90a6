"""ctypes binding of libuniprefill.so: argument marshalling only.

Every function has the name and argument order of its C entry point
(include/uniprefill.h).  Tensors are torch tensors on the GPU (device pointers)
or numpy arrays (host pointers); nothing is computed here and there is no
fallback: if the library is missing the import fails loudly.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libuniprefill.so")

UP_OK, UP_ERR_NULL, UP_ERR_SHAPE, UP_ERR_RANGE, UP_ERR_UNSUPPORTED, UP_ERR_ALIGN, UP_ERR_WORKSPACE, UP_ERR_HIP, UP_ERR_SCRATCH = range(9)
STATIC_SCRATCH_BYTES = 32 << 20
UP_BF16, UP_F32 = 0, 1

EXPORTS = ["uniprefill_plan", "uniprefill_score", "uniprefill_select", "uniprefill_compact",
           "uniprefill_scatter", "uniprefill_fused", "uniprefill_fused_phases", "uniprefill_select_top_p",
           "uniprefill_compact_counted", "uniprefill_fused_top_p", "uniprefill_compose_index",
           "uniprefill_slot_mapping", "uniprefill_plan_chunked", "uniprefill_score_chunked",
           "uniprefill_select_chunked", "uniprefill_fused_chunked", "uniprefill_compact_column", "uniprefill_seqused",
           "uniprefill_score_paged", "uniprefill_fused_paged", "uniprefill_select_top_p_chunked",
           "uniprefill_fused_top_p_chunked", "uniprefill_keep_mask", "uniprefill_fused_lse",
           "uniprefill_score_lse", "uniprefill_fused_top_p_lse", "uniprefill_score_partial",
           "uniprefill_scores_from_partials", "uniprefill_fused_static",
           "uniprefill_attention_plan", "uniprefill_attention", "uniprefill_q4_row_bytes", "uniprefill_cache_store_q4",
           "uniprefill_cache_load_q4", "uniprefill_attention_q4_plan", "uniprefill_attention_q4",
           "uniprefill_cache_evict", "uniprefill_attention_window_plan", "uniprefill_attention_window",
           "uniprefill_attention_window_step_plan", "uniprefill_attention_window_step", "uniprefill_linear_attention_plan",
           "uniprefill_linear_attention", "uniprefill_linear_attention_step", "uniprefill_norm_rotate", "uniprefill_append_pages",
           "uniprefill_append_pages_dropped",
           "uniprefill_status_string"]

UP_PHASE_PLAN, UP_PHASE_ROW_STATS, UP_PHASE_MERGE_STATS, UP_PHASE_SWEEP_SELECT, UP_PHASE_GATHER = 1, 2, 4, 8, 16
UP_PHASE_ALL = 31
UP_PHASE_GATHER_IN_SELECT = 32


class up_params(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("total_tokens", ctypes.c_int32),
        ("block_size", ctypes.c_int32), ("n_obs", ctypes.c_int32), ("n_sink", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("hidden_dim", ctypes.c_int32),
        ("q_row_stride", ctypes.c_int64), ("k_row_stride", ctypes.c_int64),
        ("hidden_row_stride", ctypes.c_int64),
        ("softmax_scale", ctypes.c_float),
        ("qk_dtype", ctypes.c_int32), ("hidden_dtype", ctypes.c_int32),
    ]


class UniPrefillError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()'). "
            "There is no fallback path.")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
    P = ctypes.POINTER(up_params)
    i64, i32, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    ws = [vp, sz]                                   # workspace, workspace_bytes
    keys = [i32p, i32p]                             # cu_seqlens_k_dev, cu_seqlens_k_host
    table = [i32p, i64, i32]                        # block_table, block_table_stride, kv_block_size
    outs = [vp, i32p, i32p, i32p, f32p]             # hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores
    lib.uniprefill_plan.argtypes = [P, i32p, f32p, i32p, ctypes.POINTER(i64), ctypes.POINTER(sz)]
    lib.uniprefill_plan_chunked.argtypes = [P, i32p, i32p, f32p, i32p, ctypes.POINTER(i64), ctypes.POINTER(sz)]
    lib.uniprefill_score.argtypes = [P, vp, vp, i32p, i32p, f32p] + ws + [vp]
    lib.uniprefill_score_chunked.argtypes = [P, vp, vp, i32p, i32p] + keys + [f32p] + ws + [vp]
    lib.uniprefill_score_paged.argtypes = [P, vp, vp, i32p, i32p] + keys + table + [f32p] + ws + [vp]
    lib.uniprefill_score_lse.argtypes = [P, vp, vp, f32p, i64, i32p, i32p] + keys + table + [f32p] + ws + [vp]
    lib.uniprefill_score_partial.argtypes = [P, vp, vp, i32p, i32p] + keys + [vp] + ws + [vp]
    lib.uniprefill_scores_from_partials.argtypes = [vp, i32, i64, i32p, i32, i32, i32, i32, f32p, vp]
    lib.uniprefill_select.argtypes = [P, f32p, i32p, i32p, f32p, f32p, i32p, i32p, vp]
    lib.uniprefill_select_chunked.argtypes = [P, f32p, i32p, i32p] + keys + [f32p, f32p, i32p, i32p, vp]
    lib.uniprefill_select_top_p.argtypes = [P, f32p, i32p, i32p, f32p, f32p, i32p, i32p] + ws + [vp]
    lib.uniprefill_select_top_p_chunked.argtypes = [P, f32p, i32p, i32p] + keys + [f32p, f32p, i32p, i32p] + ws + [vp]
    lib.uniprefill_compact.argtypes = [P, vp, i32p, i32p, i64, vp, i32p, vp]
    lib.uniprefill_compact_counted.argtypes = [P, vp, i32p, i32p, i32p, i64, vp, i32p, vp]
    lib.uniprefill_compact_column.argtypes = [vp, i32, i32p, i64, i32p, vp, vp]
    lib.uniprefill_scatter.argtypes = [P, vp, i32p, i64, vp, vp]
    fused_in = [P, vp, vp, vp, i32p, i32p, i32p]    # params, q, k, hidden, pos, cu_seqlens_dev, cu_seqlens_host
    lib.uniprefill_fused.argtypes = fused_in + [f32p, f32p] + outs + ws + [vp]
    lib.uniprefill_fused_static.argtypes = fused_in + [f32p, f32p] + outs + [vp]
    lib.uniprefill_fused_phases.argtypes = fused_in + [f32p, f32p] + outs + ws + [ctypes.c_int, vp]
    lib.uniprefill_fused_chunked.argtypes = fused_in + keys + [f32p, f32p] + outs + ws + [vp]
    lib.uniprefill_fused_paged.argtypes = fused_in + keys + table + [f32p, f32p] + outs + ws + [vp]
    lib.uniprefill_fused_top_p.argtypes = fused_in + [f32p, f32p] + outs + ws + [vp]
    lib.uniprefill_fused_top_p_chunked.argtypes = fused_in + keys + table + [f32p, f32p] + outs + ws + [vp]
    lse_in = [P, vp, vp, f32p, i64, vp, i32p, i32p, i32p]   # params, q, k, lse, lse_row_stride, hidden, pos, cu dev/host
    lib.uniprefill_fused_lse.argtypes = lse_in + keys + table + [f32p, f32p] + outs + ws + [vp]
    lib.uniprefill_fused_top_p_lse.argtypes = lse_in + keys + table + [f32p, f32p] + outs + ws + [vp]
    lib.uniprefill_compose_index.argtypes = [i32p, i64, i32p, i32p, i64, i32p, vp]
    lib.uniprefill_slot_mapping.argtypes = [i32p, i32p, i32, i32p, i64, i32, i64, vp, vp]
    lib.uniprefill_keep_mask.argtypes = [i32p, i64, i32p, i64, vp, vp]
    lib.uniprefill_seqused.argtypes = [i32p, i32, i32p, i32p, i32p, i32, i32, i32p, vp]
    lib.uniprefill_attention_plan.argtypes = [P, i32p, i32p, ctypes.POINTER(sz)]
    lib.uniprefill_attention.argtypes = [P, vp, vp, vp, i64, i32p, i32p] + keys + table + [vp, i64, f32p, i64] + ws + [vp]
    lib.uniprefill_q4_row_bytes.argtypes = [i32, i32]
    lib.uniprefill_cache_store_q4.argtypes = [P, vp, vp, i64, vp, i64, i32p, vp, vp, i64, i64, vp]
    lib.uniprefill_cache_load_q4.argtypes = [P, vp, vp, i64, i64, vp, i64, i32p, vp, vp, i64, vp]
    lib.uniprefill_attention_q4_plan.argtypes = [P, i32, i32, ctypes.POINTER(sz)]
    lib.uniprefill_attention_q4.argtypes = [P, vp, vp, vp, i64, i32p, i32] + table + [vp, i64, f32p, i64, f32p, f32p, i64] + ws + [vp]
    lib.uniprefill_cache_evict.argtypes = [vp, vp, i64, i64, f32p, i64, i32p, i32, i32, i32, i32, i32, i32p, i64, i32p, i64, i32,
                                           i32p, f32p, i64, i32p, vp]
    band, f32 = [i32, i32], ctypes.c_float          # window, n_sink
    lib.uniprefill_attention_window_plan.argtypes = [P, i32p, i32p] + band + [ctypes.POINTER(sz)]
    lib.uniprefill_attention_window.argtypes = [P, vp, vp, vp, i64, i32p, i32p] + keys + table + band + [vp, i64, f32p, i64] + ws + [vp]
    lib.uniprefill_attention_window_step_plan.argtypes = [P, i32] + band + [ctypes.POINTER(sz)]
    lib.uniprefill_attention_window_step.argtypes = [P, vp, vp, vp, i64, i32p, i32] + table + band + [vp, i64, f32p, i64] + ws + [vp]
    states = [f32p, f32p, i64, i64, i32p, i32p]     # log_decay, states, state_stride, num_states, state_in, state_out
    lib.uniprefill_linear_attention_plan.argtypes = [P, i32p, ctypes.POINTER(sz)]
    lib.uniprefill_linear_attention.argtypes = [P, vp, vp, vp, i64, i32p, i32p] + states + [vp, i64] + ws + [vp]
    lib.uniprefill_linear_attention_step.argtypes = [P, vp, vp, vp, i64] + states + [vp, i64, vp]
    lib.uniprefill_norm_rotate.argtypes = [P, vp, vp, vp, i64, vp, vp, f32, i32p, f32p, i32, i32, i32p, vp, i64, vp, i64, vp, i64, vp, i64,
                                           vp]
    pages = [i32, i32, i32p, i64, i32p, i32p, i32p, i32p, i32p, i32p, i32p, vp, i64, i32p, vp]
    lib.uniprefill_append_pages.argtypes = [i32p, i32p] + pages
    lib.uniprefill_append_pages_dropped.argtypes = [i32p, i32p, i32p] + pages
    for name in EXPORTS[:-1]:
        getattr(lib, name).restype = ctypes.c_int
    lib.uniprefill_q4_row_bytes.restype = i64
    lib.uniprefill_status_string.argtypes = [ctypes.c_int]
    lib.uniprefill_status_string.restype = ctypes.c_char_p
    return lib


_lib = _load()


def lib():
    """The loaded ctypes library (for tests that poke the raw C ABI)."""
    return _lib


def status_string(status: int) -> str:
    return _lib.uniprefill_status_string(int(status)).decode()


def ptr(x):
    """Address of a torch tensor / numpy array / int / None as a void*."""
    if x is None:
        return None
    if isinstance(x, int):
        return ctypes.c_void_p(x)
    if isinstance(x, np.ndarray):
        return ctypes.c_void_p(x.ctypes.data)
    return ctypes.c_void_p(x.data_ptr())      # torch tensor


def _addr(x):
    """ptr without the c_void_p object, which the declared argument types do not need: 0.2 instead of 0.4 us an argument, and the calls
    of a decode step have fifteen."""
    if x is None:
        return None
    try:
        return x.data_ptr()
    except AttributeError:
        return x if isinstance(x, int) else x.ctypes.data


def _stream(stream):
    if stream is None:
        import torch
        # torch.cuda.current_stream().cuda_stream without the Stream object: 0.3 instead of 2.7 us of a call's 8.  The function is not
        # part of torch's public interface: where a release lacks it, the public way.
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device()))
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _check(status: int, where: str, check: bool):
    if check and status != UP_OK:
        raise UniPrefillError(status, where)
    return status


def make_params(*, num_seqs, total_tokens, block_size, n_obs=128, n_sink=128, num_q_heads=0,
                num_kv_heads=0, head_dim=128, hidden_dim=0, q_row_stride=None, k_row_stride=None,
                hidden_row_stride=None, softmax_scale=0.0, qk_dtype=UP_BF16, hidden_dtype=UP_BF16) -> up_params:
    return up_params(
        num_seqs, total_tokens, block_size, n_obs, n_sink, num_q_heads, num_kv_heads, head_dim, hidden_dim,
        num_q_heads * head_dim if q_row_stride is None else q_row_stride,
        num_kv_heads * head_dim if k_row_stride is None else k_row_stride,
        hidden_dim if hidden_row_stride is None else hidden_row_stride,
        softmax_scale, qk_dtype, hidden_dtype)


def uniprefill_plan(p: up_params, cu_seqlens_host: np.ndarray, keep_ratio_host: np.ndarray, *,
                    want_workspace: bool = True, check: bool = True):
    """Returns (status, new_cu_seqlens_host, total_kept, workspace_bytes)."""
    new_cu = np.zeros(p.num_seqs + 1, dtype=np.int32)
    total = ctypes.c_int64(0)
    ws = ctypes.c_size_t(0)
    st = _lib.uniprefill_plan(ctypes.byref(p), ptr(cu_seqlens_host), ptr(keep_ratio_host), ptr(new_cu),
                              ctypes.byref(total), ctypes.byref(ws) if want_workspace else None)
    _check(st, "uniprefill_plan", check)
    return st, new_cu, int(total.value), int(ws.value)


def uniprefill_score(p, q, k, cu_seqlens_dev, cu_seqlens_host, scores_out, workspace, workspace_bytes,
                     stream=None, check=True):
    st = _lib.uniprefill_score(ctypes.byref(p), ptr(q), ptr(k), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                               ptr(scores_out), ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_score", check)


def uniprefill_select(p, scores, cu_seqlens_dev, cu_seqlens_host, keep_ratio_dev, keep_ratio_host,
                      kept_idx, new_cu_seqlens_dev, stream=None, check=True):
    st = _lib.uniprefill_select(ctypes.byref(p), ptr(scores), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                                ptr(keep_ratio_dev), ptr(keep_ratio_host), ptr(kept_idx),
                                ptr(new_cu_seqlens_dev), _stream(stream))
    return _check(st, "uniprefill_select", check)


def uniprefill_compact(p, hidden, pos, kept_idx, total_kept, hidden_out, pos_out, stream=None, check=True):
    st = _lib.uniprefill_compact(ctypes.byref(p), ptr(hidden), ptr(pos), ptr(kept_idx), int(total_kept),
                                 ptr(hidden_out), ptr(pos_out), _stream(stream))
    return _check(st, "uniprefill_compact", check)


def uniprefill_scatter(p, hidden_compact, kept_idx, total_kept, hidden_full_inout, stream=None, check=True):
    st = _lib.uniprefill_scatter(ctypes.byref(p), ptr(hidden_compact), ptr(kept_idx), int(total_kept),
                                 ptr(hidden_full_inout), _stream(stream))
    return _check(st, "uniprefill_scatter", check)


def uniprefill_fused(p, q, k, hidden, pos, cu_seqlens_dev, cu_seqlens_host, keep_ratio_dev, keep_ratio_host,
                     hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores_out, workspace,
                     workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_fused(ctypes.byref(p), ptr(q), ptr(k), ptr(hidden), ptr(pos), ptr(cu_seqlens_dev),
                               ptr(cu_seqlens_host), ptr(keep_ratio_dev), ptr(keep_ratio_host),
                               ptr(hidden_out), ptr(pos_out), ptr(kept_idx), ptr(new_cu_seqlens_dev),
                               ptr(scores_out), ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_fused", check)


def uniprefill_fused_static(p, q, k, hidden, pos, cu_seqlens_dev, cu_seqlens_host, keep_ratio_dev, keep_ratio_host,
                            hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores_out, stream=None, check=True):
    st = _lib.uniprefill_fused_static(ctypes.byref(p), ptr(q), ptr(k), ptr(hidden), ptr(pos), ptr(cu_seqlens_dev),
                                      ptr(cu_seqlens_host), ptr(keep_ratio_dev), ptr(keep_ratio_host),
                                      ptr(hidden_out), ptr(pos_out), ptr(kept_idx), ptr(new_cu_seqlens_dev),
                                      ptr(scores_out), _stream(stream))
    return _check(st, "uniprefill_fused_static", check)


def uniprefill_compact_column(column, elem_bytes, kept_idx, capacity, total_kept_dev, column_out, stream=None,
                              check=True):
    st = _lib.uniprefill_compact_column(ptr(column), int(elem_bytes), ptr(kept_idx), ctypes.c_int64(capacity),
                                        ptr(total_kept_dev), ptr(column_out), _stream(stream))
    return _check(st, "uniprefill_compact_column", check)


def uniprefill_fused_lse(p, q, k, lse, lse_row_stride, hidden, pos, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev,
                         cu_seqlens_k_host, block_table, block_table_stride, kv_block_size, keep_ratio_dev,
                         keep_ratio_host, hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores_out, workspace,
                         workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_fused_lse(ctypes.byref(p), ptr(q), ptr(k), ptr(lse), ctypes.c_int64(lse_row_stride), ptr(hidden),
                                   ptr(pos), ptr(cu_seqlens_dev), ptr(cu_seqlens_host), ptr(cu_seqlens_k_dev),
                                   ptr(cu_seqlens_k_host), ptr(block_table), ctypes.c_int64(block_table_stride),
                                   int(kv_block_size), ptr(keep_ratio_dev), ptr(keep_ratio_host), ptr(hidden_out),
                                   ptr(pos_out), ptr(kept_idx), ptr(new_cu_seqlens_dev), ptr(scores_out),
                                   ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_fused_lse", check)


def uniprefill_score_lse(p, q, k, lse, lse_row_stride, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev,
                         cu_seqlens_k_host, block_table, block_table_stride, kv_block_size, scores_out, workspace,
                         workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_score_lse(ctypes.byref(p), ptr(q), ptr(k), ptr(lse), ctypes.c_int64(lse_row_stride),
                                   ptr(cu_seqlens_dev), ptr(cu_seqlens_host), ptr(cu_seqlens_k_dev),
                                   ptr(cu_seqlens_k_host), ptr(block_table), ctypes.c_int64(block_table_stride),
                                   int(kv_block_size), ptr(scores_out), ptr(workspace), workspace_bytes,
                                   _stream(stream))
    return _check(st, "uniprefill_score_lse", check)


def uniprefill_fused_top_p_lse(p, q, k, lse, lse_row_stride, hidden, pos, cu_seqlens_dev, cu_seqlens_host,
                               cu_seqlens_k_dev, cu_seqlens_k_host, block_table, block_table_stride, kv_block_size,
                               top_p_dev, top_p_host, hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores,
                               workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_fused_top_p_lse(ctypes.byref(p), ptr(q), ptr(k), ptr(lse), ctypes.c_int64(lse_row_stride),
                                         ptr(hidden), ptr(pos), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                                         ptr(cu_seqlens_k_dev), ptr(cu_seqlens_k_host), ptr(block_table),
                                         ctypes.c_int64(block_table_stride), int(kv_block_size), ptr(top_p_dev),
                                         ptr(top_p_host), ptr(hidden_out), ptr(pos_out), ptr(kept_idx),
                                         ptr(new_cu_seqlens_dev), ptr(scores), ptr(workspace), workspace_bytes,
                                         _stream(stream))
    return _check(st, "uniprefill_fused_top_p_lse", check)


def uniprefill_score_partial(p, q, k, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host, colsum_out,
                             workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_score_partial(ctypes.byref(p), ptr(q), ptr(k), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                                       ptr(cu_seqlens_k_dev), ptr(cu_seqlens_k_host), ptr(colsum_out), ptr(workspace),
                                       workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_score_partial", check)


def uniprefill_scores_from_partials(partials, num_parts, part_stride, cu_seqlens_dev, num_seqs, total_tokens, n_obs,
                                    total_q_heads, scores_out, stream=None, check=True):
    st = _lib.uniprefill_scores_from_partials(ptr(partials), int(num_parts), ctypes.c_int64(part_stride),
                                              ptr(cu_seqlens_dev), int(num_seqs), int(total_tokens), int(n_obs),
                                              int(total_q_heads), ptr(scores_out), _stream(stream))
    return _check(st, "uniprefill_scores_from_partials", check)


def uniprefill_keep_mask(kept_idx, capacity, total_kept_dev, total_tokens, mask_out, stream=None, check=True):
    st = _lib.uniprefill_keep_mask(ptr(kept_idx), ctypes.c_int64(capacity), ptr(total_kept_dev),
                                   ctypes.c_int64(total_tokens), ptr(mask_out), _stream(stream))
    return _check(st, "uniprefill_keep_mask", check)


def uniprefill_seqused(drop_layers_host, retained_dev, kv_len_dev, orig_len_dev, num_seqs, num_layers, seqused_out,
                       stream=None, check=True):
    layers = np.ascontiguousarray(drop_layers_host, dtype=np.int32)
    st = _lib.uniprefill_seqused(ptr(layers), int(layers.shape[0]), ptr(retained_dev), ptr(kv_len_dev),
                                 ptr(orig_len_dev), int(num_seqs), int(num_layers), ptr(seqused_out),
                                 _stream(stream))
    return _check(st, "uniprefill_seqused", check)


def uniprefill_plan_chunked(p: up_params, cu_seqlens_host: np.ndarray, cu_seqlens_k_host: np.ndarray,
                            keep_ratio_host: np.ndarray, *, want_workspace: bool = True, check: bool = True):
    """Returns (status, new_cu_seqlens_host, total_kept, workspace_bytes)."""
    new_cu = np.zeros(p.num_seqs + 1, dtype=np.int32)
    total = ctypes.c_int64(0)
    ws = ctypes.c_size_t(0)
    st = _lib.uniprefill_plan_chunked(ctypes.byref(p), ptr(cu_seqlens_host), ptr(cu_seqlens_k_host),
                                      ptr(keep_ratio_host), ptr(new_cu), ctypes.byref(total),
                                      ctypes.byref(ws) if want_workspace else None)
    _check(st, "uniprefill_plan_chunked", check)
    return st, new_cu, int(total.value), int(ws.value)


def uniprefill_score_chunked(p, q, k, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                             scores_out, workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_score_chunked(ctypes.byref(p), ptr(q), ptr(k), ptr(cu_seqlens_dev),
                                       ptr(cu_seqlens_host), ptr(cu_seqlens_k_dev), ptr(cu_seqlens_k_host),
                                       ptr(scores_out), ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_score_chunked", check)


def uniprefill_select_chunked(p, scores, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                              keep_ratio_dev, keep_ratio_host, kept_idx, new_cu_seqlens_dev, stream=None,
                              check=True):
    st = _lib.uniprefill_select_chunked(ctypes.byref(p), ptr(scores), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                                        ptr(cu_seqlens_k_dev), ptr(cu_seqlens_k_host), ptr(keep_ratio_dev),
                                        ptr(keep_ratio_host), ptr(kept_idx), ptr(new_cu_seqlens_dev),
                                        _stream(stream))
    return _check(st, "uniprefill_select_chunked", check)


def uniprefill_fused_chunked(p, q, k, hidden, pos, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev,
                             cu_seqlens_k_host, keep_ratio_dev, keep_ratio_host, hidden_out, pos_out, kept_idx,
                             new_cu_seqlens_dev, scores_out, workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_fused_chunked(ctypes.byref(p), ptr(q), ptr(k), ptr(hidden), ptr(pos),
                                       ptr(cu_seqlens_dev), ptr(cu_seqlens_host), ptr(cu_seqlens_k_dev),
                                       ptr(cu_seqlens_k_host), ptr(keep_ratio_dev), ptr(keep_ratio_host),
                                       ptr(hidden_out), ptr(pos_out), ptr(kept_idx), ptr(new_cu_seqlens_dev),
                                       ptr(scores_out), ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_fused_chunked", check)


def uniprefill_score_paged(p, q, k_cache, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                           block_table, block_table_stride, kv_block_size, scores_out, workspace, workspace_bytes,
                           stream=None, check=True):
    st = _lib.uniprefill_score_paged(ctypes.byref(p), ptr(q), ptr(k_cache), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                                     ptr(cu_seqlens_k_dev), ptr(cu_seqlens_k_host), ptr(block_table),
                                     ctypes.c_int64(block_table_stride), int(kv_block_size), ptr(scores_out),
                                     ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_score_paged", check)


def uniprefill_fused_paged(p, q, k_cache, hidden, pos, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev,
                           cu_seqlens_k_host, block_table, block_table_stride, kv_block_size, keep_ratio_dev,
                           keep_ratio_host, hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores_out, workspace,
                           workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_fused_paged(ctypes.byref(p), ptr(q), ptr(k_cache), ptr(hidden), ptr(pos),
                                     ptr(cu_seqlens_dev), ptr(cu_seqlens_host), ptr(cu_seqlens_k_dev),
                                     ptr(cu_seqlens_k_host), ptr(block_table), ctypes.c_int64(block_table_stride),
                                     int(kv_block_size), ptr(keep_ratio_dev), ptr(keep_ratio_host), ptr(hidden_out),
                                     ptr(pos_out), ptr(kept_idx), ptr(new_cu_seqlens_dev), ptr(scores_out),
                                     ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_fused_paged", check)


def uniprefill_select_top_p_chunked(p, scores, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                                    top_p_dev, top_p_host, kept_idx, new_cu_seqlens_dev, workspace, workspace_bytes,
                                    stream=None, check=True):
    st = _lib.uniprefill_select_top_p_chunked(ctypes.byref(p), ptr(scores), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                                              ptr(cu_seqlens_k_dev), ptr(cu_seqlens_k_host), ptr(top_p_dev),
                                              ptr(top_p_host), ptr(kept_idx), ptr(new_cu_seqlens_dev), ptr(workspace),
                                              workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_select_top_p_chunked", check)


def uniprefill_fused_top_p_chunked(p, q, k, hidden, pos, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev,
                                   cu_seqlens_k_host, block_table, block_table_stride, kv_block_size, top_p_dev,
                                   top_p_host, hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores, workspace,
                                   workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_fused_top_p_chunked(ctypes.byref(p), ptr(q), ptr(k), ptr(hidden), ptr(pos),
                                             ptr(cu_seqlens_dev), ptr(cu_seqlens_host), ptr(cu_seqlens_k_dev),
                                             ptr(cu_seqlens_k_host), ptr(block_table),
                                             ctypes.c_int64(block_table_stride), int(kv_block_size), ptr(top_p_dev),
                                             ptr(top_p_host), ptr(hidden_out), ptr(pos_out), ptr(kept_idx),
                                             ptr(new_cu_seqlens_dev), ptr(scores), ptr(workspace), workspace_bytes,
                                             _stream(stream))
    return _check(st, "uniprefill_fused_top_p_chunked", check)


def uniprefill_fused_phases(p, q, k, hidden, pos, cu_seqlens_dev, cu_seqlens_host, keep_ratio_dev,
                            keep_ratio_host, hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores_out,
                            workspace, workspace_bytes, phase_mask, stream=None, check=True):
    st = _lib.uniprefill_fused_phases(ctypes.byref(p), ptr(q), ptr(k), ptr(hidden), ptr(pos),
                                      ptr(cu_seqlens_dev), ptr(cu_seqlens_host), ptr(keep_ratio_dev),
                                      ptr(keep_ratio_host), ptr(hidden_out), ptr(pos_out), ptr(kept_idx),
                                      ptr(new_cu_seqlens_dev), ptr(scores_out), ptr(workspace),
                                      workspace_bytes, int(phase_mask), _stream(stream))
    return _check(st, "uniprefill_fused_phases", check)


def uniprefill_select_top_p(p, scores, cu_seqlens_dev, cu_seqlens_host, top_p_dev, top_p_host, kept_idx,
                            new_cu_seqlens_dev, workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_select_top_p(ctypes.byref(p), ptr(scores), ptr(cu_seqlens_dev), ptr(cu_seqlens_host),
                                      ptr(top_p_dev), ptr(top_p_host), ptr(kept_idx), ptr(new_cu_seqlens_dev),
                                      ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_select_top_p", check)


def uniprefill_compact_counted(p, hidden, pos, kept_idx, total_kept_dev, capacity, hidden_out, pos_out,
                               stream=None, check=True):
    st = _lib.uniprefill_compact_counted(ctypes.byref(p), ptr(hidden), ptr(pos), ptr(kept_idx),
                                         ptr(total_kept_dev), int(capacity), ptr(hidden_out), ptr(pos_out),
                                         _stream(stream))
    return _check(st, "uniprefill_compact_counted", check)


def uniprefill_fused_top_p(p, q, k, hidden, pos, cu_seqlens_dev, cu_seqlens_host, top_p_dev, top_p_host,
                           hidden_out, pos_out, kept_idx, new_cu_seqlens_dev, scores, workspace,
                           workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_fused_top_p(ctypes.byref(p), ptr(q), ptr(k), ptr(hidden), ptr(pos),
                                     ptr(cu_seqlens_dev), ptr(cu_seqlens_host), ptr(top_p_dev),
                                     ptr(top_p_host), ptr(hidden_out), ptr(pos_out), ptr(kept_idx),
                                     ptr(new_cu_seqlens_dev), ptr(scores), ptr(workspace), workspace_bytes,
                                     _stream(stream))
    return _check(st, "uniprefill_fused_top_p", check)


def uniprefill_compose_index(outer_idx, n_outer, inner_idx, n_inner_dev, n_inner, composed_idx, stream=None,
                             check=True):
    st = _lib.uniprefill_compose_index(ptr(outer_idx), int(n_outer), ptr(inner_idx), ptr(n_inner_dev),
                                       int(n_inner), ptr(composed_idx), _stream(stream))
    return _check(st, "uniprefill_compose_index", check)


def uniprefill_slot_mapping(pos_kept, new_cu_seqlens_dev, num_seqs, block_table, block_table_stride,
                            kv_block_size, capacity, slots, stream=None, check=True):
    st = _lib.uniprefill_slot_mapping(ptr(pos_kept), ptr(new_cu_seqlens_dev), int(num_seqs), ptr(block_table),
                                      int(block_table_stride), int(kv_block_size), int(capacity), ptr(slots),
                                      _stream(stream))
    return _check(st, "uniprefill_slot_mapping", check)


def uniprefill_attention_plan(p: up_params, cu_seqlens_host: np.ndarray, cu_seqlens_k_host=None, *, check: bool = True):
    """Returns (status, workspace_bytes)."""
    ws = ctypes.c_size_t(0)
    st = _lib.uniprefill_attention_plan(ctypes.byref(p), ptr(cu_seqlens_host), ptr(cu_seqlens_k_host), ctypes.byref(ws))
    _check(st, "uniprefill_attention_plan", check)
    return st, int(ws.value)


def uniprefill_attention(p, q, k, v, v_row_stride, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                         block_table, block_table_stride, kv_block_size, out, out_row_stride, lse_out, lse_row_stride,
                         workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_attention(ctypes.byref(p), ptr(q), ptr(k), ptr(v), int(v_row_stride), ptr(cu_seqlens_dev),
                                   ptr(cu_seqlens_host), ptr(cu_seqlens_k_dev), ptr(cu_seqlens_k_host), ptr(block_table),
                                   int(block_table_stride), int(kv_block_size), ptr(out), int(out_row_stride), ptr(lse_out),
                                   int(lse_row_stride), ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_attention", check)


def uniprefill_q4_row_bytes(num_kv_heads, head_dim):
    return int(_lib.uniprefill_q4_row_bytes(int(num_kv_heads), int(head_dim)))


def uniprefill_cache_store_q4(p, k, v, v_row_stride, slots, n, count_dev, k_cache, v_cache, cache_row_stride, num_slots,
                              stream=None, check=True):
    st = _lib.uniprefill_cache_store_q4(ctypes.byref(p), ptr(k), ptr(v), int(v_row_stride), ptr(slots), int(n),
                                        ptr(count_dev), ptr(k_cache), ptr(v_cache), int(cache_row_stride), int(num_slots),
                                        _stream(stream))
    return _check(st, "uniprefill_cache_store_q4", check)


def uniprefill_cache_load_q4(p, k_cache, v_cache, cache_row_stride, num_slots, slots, n, count_dev, k_out, v_out,
                             v_row_stride, stream=None, check=True):
    st = _lib.uniprefill_cache_load_q4(ctypes.byref(p), ptr(k_cache), ptr(v_cache), int(cache_row_stride), int(num_slots),
                                       ptr(slots), int(n), ptr(count_dev), ptr(k_out), ptr(v_out), int(v_row_stride),
                                       _stream(stream))
    return _check(st, "uniprefill_cache_load_q4", check)


def uniprefill_attention_q4_plan(p: up_params, max_kv_len, want_mass, *, check: bool = True):
    """Returns (status, workspace_bytes)."""
    ws = ctypes.c_size_t(0)
    st = _lib.uniprefill_attention_q4_plan(ctypes.byref(p), int(max_kv_len), int(bool(want_mass)), ctypes.byref(ws))
    _check(st, "uniprefill_attention_q4_plan", check)
    return st, int(ws.value)


def uniprefill_attention_q4(p, q, k_cache, v_cache, cache_row_stride, kv_len_dev, max_kv_len, block_table,
                            block_table_stride, kv_block_size, out, out_row_stride, lse_out, lse_row_stride, mass_in,
                            mass_out, mass_row_stride, workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_attention_q4(ctypes.byref(p), ptr(q), ptr(k_cache), ptr(v_cache), int(cache_row_stride),
                                      ptr(kv_len_dev), int(max_kv_len), ptr(block_table), int(block_table_stride),
                                      int(kv_block_size), ptr(out), int(out_row_stride), ptr(lse_out), int(lse_row_stride),
                                      ptr(mass_in), ptr(mass_out), int(mass_row_stride), ptr(workspace), workspace_bytes,
                                      _stream(stream))
    return _check(st, "uniprefill_attention_q4", check)


def uniprefill_cache_evict(k_cache, v_cache, row_bytes, cache_row_stride, mass, mass_row_stride, kv_len_dev, num_seqs,
                           max_kv_len, budget, n_sink, n_recent, block_table, block_table_stride, new_table,
                           new_table_stride, kv_block_size, kept_idx, mass_out, mass_out_stride, new_len, stream=None,
                           check=True):
    st = _lib.uniprefill_cache_evict(ptr(k_cache), ptr(v_cache), int(row_bytes), int(cache_row_stride), ptr(mass),
                                     int(mass_row_stride), ptr(kv_len_dev), int(num_seqs), int(max_kv_len), int(budget),
                                     int(n_sink), int(n_recent), ptr(block_table), int(block_table_stride), ptr(new_table),
                                     int(new_table_stride), int(kv_block_size), ptr(kept_idx), ptr(mass_out),
                                     int(mass_out_stride), ptr(new_len), _stream(stream))
    return _check(st, "uniprefill_cache_evict", check)


def uniprefill_attention_window_plan(p: up_params, cu_seqlens_host: np.ndarray, cu_seqlens_k_host, window, n_sink, *, check: bool = True):
    """Returns (status, workspace_bytes)."""
    ws = ctypes.c_size_t(0)
    st = _lib.uniprefill_attention_window_plan(ctypes.byref(p), _addr(cu_seqlens_host), _addr(cu_seqlens_k_host), int(window), int(n_sink),
                                               ctypes.byref(ws))
    _check(st, "uniprefill_attention_window_plan", check)
    return st, int(ws.value)


def uniprefill_attention_window(p, q, k, v, v_row_stride, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                                block_table, block_table_stride, kv_block_size, window, n_sink, out, out_row_stride, lse_out,
                                lse_row_stride, workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_attention_window(ctypes.byref(p), _addr(q), _addr(k), _addr(v), int(v_row_stride), _addr(cu_seqlens_dev),
                                          _addr(cu_seqlens_host), _addr(cu_seqlens_k_dev), _addr(cu_seqlens_k_host), _addr(block_table),
                                          int(block_table_stride), int(kv_block_size), int(window), int(n_sink), _addr(out),
                                          int(out_row_stride), _addr(lse_out), int(lse_row_stride), _addr(workspace), workspace_bytes,
                                          _stream(stream))
    return _check(st, "uniprefill_attention_window", check)


def uniprefill_attention_window_step_plan(p: up_params, max_kv_len, window, n_sink, *, check: bool = True):
    """Returns (status, workspace_bytes)."""
    ws = ctypes.c_size_t(0)
    st = _lib.uniprefill_attention_window_step_plan(ctypes.byref(p), int(max_kv_len), int(window), int(n_sink), ctypes.byref(ws))
    _check(st, "uniprefill_attention_window_step_plan", check)
    return st, int(ws.value)


def uniprefill_attention_window_step(p, q, k_cache, v_cache, v_row_stride, kv_len_dev, max_kv_len, block_table, block_table_stride,
                                     kv_block_size, window, n_sink, out, out_row_stride, lse_out, lse_row_stride, workspace,
                                     workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_attention_window_step(ctypes.byref(p), _addr(q), _addr(k_cache), _addr(v_cache), int(v_row_stride),
                                               _addr(kv_len_dev), int(max_kv_len), _addr(block_table), int(block_table_stride),
                                               int(kv_block_size), int(window), int(n_sink), _addr(out), int(out_row_stride),
                                               _addr(lse_out), int(lse_row_stride), _addr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_attention_window_step", check)


def uniprefill_linear_attention_plan(p: up_params, cu_seqlens_host: np.ndarray, *, check: bool = True):
    """Returns (status, workspace_bytes)."""
    ws = ctypes.c_size_t(0)
    st = _lib.uniprefill_linear_attention_plan(ctypes.byref(p), _addr(cu_seqlens_host), ctypes.byref(ws))
    _check(st, "uniprefill_linear_attention_plan", check)
    return st, int(ws.value)


def uniprefill_linear_attention(p, q, k, v, v_row_stride, cu_seqlens_dev, cu_seqlens_host, log_decay, states, state_stride, num_states,
                                state_in, state_out, out, out_row_stride, workspace, workspace_bytes, stream=None, check=True):
    st = _lib.uniprefill_linear_attention(ctypes.byref(p), _addr(q), _addr(k), _addr(v), int(v_row_stride), _addr(cu_seqlens_dev),
                                          _addr(cu_seqlens_host), _addr(log_decay), _addr(states), int(state_stride), int(num_states),
                                          _addr(state_in), _addr(state_out), _addr(out), int(out_row_stride), _addr(workspace),
                                          workspace_bytes, _stream(stream))
    return _check(st, "uniprefill_linear_attention", check)


def uniprefill_linear_attention_step(p, q, k, v, v_row_stride, log_decay, states, state_stride, num_states, state_in, state_out, out,
                                     out_row_stride, stream=None, check=True):
    st = _lib.uniprefill_linear_attention_step(ctypes.byref(p), _addr(q), _addr(k), _addr(v), int(v_row_stride), _addr(log_decay), _addr(states),
                                               int(state_stride), int(num_states), _addr(state_in), _addr(state_out), _addr(out),
                                               int(out_row_stride), _stream(stream))
    return _check(st, "uniprefill_linear_attention_step", check)


def uniprefill_norm_rotate(p, q, k, v, v_row_stride, q_weight, k_weight, eps, pos, inv_freq, rot_dim, pairs, count_dev, q_out,
                           q_out_row_stride, k_out, k_out_row_stride, v_out, v_out_row_stride, slots, num_slots, stream=None,
                           check=True):
    st = _lib.uniprefill_norm_rotate(ctypes.byref(p), _addr(q), _addr(k), _addr(v), int(v_row_stride), _addr(q_weight), _addr(k_weight),
                                     float(eps), _addr(pos), _addr(inv_freq), int(rot_dim), int(pairs), _addr(count_dev), _addr(q_out),
                                     int(q_out_row_stride), _addr(k_out), int(k_out_row_stride), _addr(v_out), int(v_out_row_stride),
                                     _addr(slots), int(num_slots), _stream(stream))
    return _check(st, "uniprefill_norm_rotate", check)


def uniprefill_append_pages(kv_len_dev, num_new_dev, num_seqs, kv_block_size, block_table, block_table_stride, free_pages,
                            num_free_dev, free_left_dev, new_len_dev, cu_seqlens_dev, cu_seqlens_k_dev, pos, slots, capacity,
                            num_served_dev, stream=None, check=True):
    st = _lib.uniprefill_append_pages(_addr(kv_len_dev), _addr(num_new_dev), int(num_seqs), int(kv_block_size), _addr(block_table),
                                      int(block_table_stride), _addr(free_pages), _addr(num_free_dev), _addr(free_left_dev),
                                      _addr(new_len_dev), _addr(cu_seqlens_dev), _addr(cu_seqlens_k_dev), _addr(pos), _addr(slots),
                                      int(capacity), _addr(num_served_dev), _stream(stream))
    return _check(st, "uniprefill_append_pages", check)


def uniprefill_append_pages_dropped(kv_len_dev, num_new_dev, num_dropped_dev, num_seqs, kv_block_size, block_table, block_table_stride,
                                    free_pages, num_free_dev, free_left_dev, new_len_dev, cu_seqlens_dev, cu_seqlens_k_dev, pos, slots,
                                    capacity, num_served_dev, stream=None, check=True):
    st = _lib.uniprefill_append_pages_dropped(_addr(kv_len_dev), _addr(num_new_dev), _addr(num_dropped_dev), int(num_seqs),
                                              int(kv_block_size), _addr(block_table), int(block_table_stride), _addr(free_pages),
                                              _addr(num_free_dev), _addr(free_left_dev), _addr(new_len_dev), _addr(cu_seqlens_dev),
                                              _addr(cu_seqlens_k_dev), _addr(pos), _addr(slots), int(capacity), _addr(num_served_dev),
                                              _stream(stream))
    return _check(st, "uniprefill_append_pages_dropped", check)
