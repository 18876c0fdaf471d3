"""Thin ctypes binding of the C-ABI in include/litevlm_select.h.

Argument marshalling only: torch tensors give device pointers and the current
CUDA stream; every step of the path runs in liblitevlm_select.so. There is no
CPU fallback: if the library is missing the import of this module fails. The hot
calls convert their arguments in a small CPython extension (_fastcall.so, built
with the library); the others go through ctypes.

Names follow the C functions: create / destroy / score / topk / compact /
check_device (litevlm_select_*), plus ``Selector``, a small object that owns
a handle and allocates outputs with torch.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# LITEVLM_LIB may name another build of the library (e.g. the debug variant,
# liblitevlm_select_debug.so); by default the release build in the package
LIB_PATH = os.environ.get("LITEVLM_LIB") or os.path.join(_PKG, "liblitevlm_select.so")

STATUS = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "WORKSPACE", 4: "CUDA", 5: "TIMEOUT",
          6: "DEVICE_BOUNDS"}
DTYPES = {"bf16": 0, "e4m3": 1}


class Cache(ctypes.Structure):
    """litevlm_cache_t"""
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


class Bounds(ctypes.Structure):
    """litevlm_key_bounds_t"""
    _fields_ = [("codes", ctypes.c_void_p), ("exps", ctypes.c_void_p), ("num_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32)]


class LitevlmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status
        self.name = STATUS.get(status, str(status))


class Config(ctypes.Structure):
    _fields_ = [("max_batch", ctypes.c_int32), ("max_total_visual", ctypes.c_int64),
                ("max_total_text", ctypes.c_int64), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("qk_dtype", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() (needs nvcc)")
    lib = ctypes.CDLL(LIB_PATH)
    P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.litevlm_select_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(P)]
    lib.litevlm_select_destroy.argtypes = [P]
    lib.litevlm_select_last_error.argtypes = [P]
    lib.litevlm_select_last_error.restype = ctypes.c_char_p
    lib.litevlm_select_last_launches.argtypes = [P]
    lib.litevlm_select_last_launches.restype = ctypes.c_int32
    lib.litevlm_status_string.argtypes = [ctypes.c_int]
    lib.litevlm_status_string.restype = ctypes.c_char_p
    lib.litevlm_select_score.argtypes = [P, i32, P, P, P, P, P, P, f32, f32, P, P]
    lib.litevlm_select_score_full_keys.argtypes = [P, i32, P, P, P, P, P, P, P, P, P, P, f32, f32, P, P]
    lib.litevlm_select_views.argtypes = [P, i32, i32, P, P, P, f32, f32, f32, i32, P, P, P, P, P, P]
    lib.litevlm_select_fold_norm.argtypes = [P, i32, i32, P, P, P, P]
    lib.litevlm_select_rope_table.argtypes = [P, i32, i32, f32, P, P]
    lib.litevlm_select_project.argtypes = [P, i64, i32, i32, P, P, P, f32, i32, P, P, i32, f32, P, P]
    lib.litevlm_select_topk.argtypes = [P, i32, P, P, P, P, P, f32, P, P, P, P]
    lib.litevlm_select_compact.argtypes = [P, i64, P, i64, i32, P, P, P, P]
    lib.litevlm_select_score_topk.argtypes = [P, i32, P, P, P, P, P, P, f32, f32, P, P, P, f32, P, P, P, P]
    lib.litevlm_select_check_device.argtypes = [P, P]
    lib.litevlm_select_host_view.argtypes = [P, P, ctypes.POINTER(P)]
    lib.litevlm_select_score_plan.argtypes = [P, i32, P, P, P]
    lib.litevlm_select_splice.argtypes = [P, i32, P, P, P, P, P, P, P, P, P, P, P, P, i64, P, P, P, P, P]
    lib.litevlm_select_score_noalloc.argtypes = [i32, i32, i32, i32, i32, P, P, P, P, P, P, f32, f32, P, P, P]
    lib.litevlm_select_keep_offsets.argtypes = [i32, P, P, f32, P]
    lib.litevlm_select_cache_append.argtypes = [P, i32, P, P, i32, P, P, i64, P, i64, i64, P, P, P, f32, f32, P, P, P,
                                                P, P]
    lib.litevlm_select_cache_append_granted.argtypes = [*lib.litevlm_select_cache_append.argtypes[:-2], P, P, P]
    lib.litevlm_select_cache_attend_workspace.argtypes = [P, i32, P, i32, i32, ctypes.POINTER(i64)]
    lib.litevlm_select_cache_attend.argtypes = [P, i32, P, P, i32, P, P, i64, P, P, i32, f32, P, P, P, P, i64, P]
    lib.litevlm_select_cache_evict.argtypes = [P, i32, P, P, i32, P, i32, i32, i32, i32, P, i32, P, P, P, P]
    lib.litevlm_select_verify.argtypes = [P, i32, i32, i32, P, P, P, P, P, P, P, P, P, P]
    lib.litevlm_select_cache_reserve.argtypes = [P, i32, i32, P, i32, P, P, P, i32, P, P, P, P, P, P, P]
    lib.litevlm_select_cache_bounds.argtypes = [P, i32, P, P, P, i32, P, P, P, P]
    lib.litevlm_select_cache_pick_workspace.argtypes = [P, i32, P, i32, i32, i32, ctypes.POINTER(i64)]
    lib.litevlm_select_cache_pick.argtypes = [P, i32, P, P, i32, P, P, i64, P, P, i32, i32, i32, i32, P, P, i64, P]
    lib.litevlm_select_cache_attend_picked_workspace.argtypes = [P, i32, P, i32, i32, i32, ctypes.POINTER(i64)]
    lib.litevlm_select_cache_attend_picked.argtypes = [P, i32, P, P, i32, P, P, i64, P, P, P, i32, f32, P, P, i64, P]
    lib.litevlm_select_set_wait_budget.argtypes = [P, i64]
    lib.litevlm_select_set_debug_flags.argtypes = [P, i32]
    for fn in ("create", "destroy", "score", "score_full_keys", "topk", "compact", "check_device", "score_plan",
               "score_noalloc", "splice", "views", "fold_norm", "rope_table", "project", "score_topk", "host_view",
               "keep_offsets", "cache_append", "cache_attend_workspace", "cache_attend", "cache_evict", "verify",
               "cache_reserve", "cache_bounds", "cache_pick_workspace", "cache_pick", "cache_attend_picked_workspace",
               "cache_attend_picked", "cache_append_granted", "set_wait_budget", "set_debug_flags"):
        getattr(lib, "litevlm_select_" + fn).restype = ctypes.c_int
    return lib


LIB = _load()

# every symbol declared in include/litevlm_select.h
EXPORTS = ["litevlm_select_create", "litevlm_select_destroy", "litevlm_select_last_error",
           "litevlm_status_string", "litevlm_select_score", "litevlm_select_topk", "litevlm_select_compact",
           "litevlm_select_check_device", "litevlm_select_score_plan", "litevlm_select_score_noalloc",
           "litevlm_select_splice", "litevlm_select_score_full_keys", "litevlm_select_views",
           "litevlm_select_fold_norm", "litevlm_select_rope_table", "litevlm_select_project",
           "litevlm_select_last_launches", "litevlm_select_score_topk", "litevlm_select_host_view",
           "litevlm_select_keep_offsets", "litevlm_select_cache_append", "litevlm_select_cache_attend_workspace",
           "litevlm_select_cache_attend", "litevlm_select_cache_evict", "litevlm_select_verify",
           "litevlm_select_cache_reserve", "litevlm_select_cache_bounds", "litevlm_select_cache_pick_workspace",
           "litevlm_select_cache_pick", "litevlm_select_cache_attend_picked_workspace",
           "litevlm_select_cache_attend_picked", "litevlm_select_cache_append_granted", "litevlm_select_set_wait_budget",
           "litevlm_select_set_debug_flags"]
FLAGS = {"auto": 0, "reread": 1, "resident": 2, "resident_1buf": 8, "resident_2buf": 16, "resident_flat": 64}
# LITEVLM_FLAG_SCORE_SPLIT_QUERIES: resident plans for T > 64 run each head's text rows as two pseudo-heads
QUERY_SPLIT = {"whole": 0, "split": 128}
KERNELS = {1: "score_tc (K re-read per pass)", 2: "score_res (logits resident in TMEM, one head at a time)",
           3: "score_res (logits resident in TMEM, two heads overlapped)",
           4: "score_res (logits resident in TMEM, one head at a time, flattened (request, head) schedule over "
              "every cluster that fits at once)"}
KERNELS.update({k + 3: v + ", each head's text rows as two pseudo-heads" for k, v in list(KERNELS.items())[1:]})


def _check(rc: int, handle) -> None:
    if rc != 0:
        msg = LIB.litevlm_select_last_error(handle)
        raise LitevlmError(rc, (msg or b"").decode())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _host_i32(a) -> Optional[np.ndarray]:
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        return np.ascontiguousarray(a, dtype=np.int32)
    try:
        import torch
        if isinstance(a, torch.Tensor):
            return np.ascontiguousarray(a.detach().cpu().numpy(), dtype=np.int32)
    except ImportError:
        pass
    return np.ascontiguousarray(np.asarray(a), dtype=np.int32)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        if torch.cuda.is_initialized():  # (the raw stream: torch.cuda.current_stream() takes 3 to 6 us)
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_CTYPES = {"h": ctypes.c_void_p, "i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float}


def _ctypes_value(o, kind: str):
    """What a ctypes object stands for, where an argument of the kind takes one."""
    t = _CTYPES[kind]
    if not isinstance(o, t):
        raise TypeError(f"{type(o).__name__} is no argument of type {t.__name__}")
    return 0 if o.value is None else o.value


def _load_fastcall():
    try:
        from . import _fastcall
    except ImportError as e:
        raise ImportError(f"_fastcall.so is not built; run __graft_entry__.build() ({e})") from e
    _fastcall.bind({n: ctypes.cast(getattr(LIB, "litevlm_select_" + n), ctypes.c_void_p).value
                    for n in ("score", "score_full_keys", "score_topk", "topk", "compact", "splice", "project",
                              "keep_offsets", "cache_append", "cache_attend_workspace", "cache_attend", "cache_evict",
                              "verify", "cache_reserve", "cache_bounds", "cache_pick_workspace", "cache_pick",
                              "cache_attend_picked_workspace", "cache_attend_picked", "cache_append_granted")},
                   _host_i32, np.ndarray, _ctypes_value)
    return _fastcall


_FC = _load_fastcall()


# ----------------------------------------------------------------------------
# C functions, one to one
# ----------------------------------------------------------------------------

QUERY_LAST_TOKEN = 32


def create(max_batch: int, max_total_visual: int, max_total_text: int, num_q_heads: int, num_kv_heads: int,
           head_dim: int, qk_dtype: str = "bf16", score_kernel: str = "auto", query: str = "all",
           query_split: str = "whole") -> int:
    """query: "all" (every text token is a query) or "last" (only the last one).
    query_split: "whole", or "split" (resident plans for T > 64 run each head's
    text rows as two pseudo-heads)."""
    cfg = Config(max_batch, max_total_visual, max_total_text, num_q_heads, num_kv_heads, head_dim,
                 DTYPES[qk_dtype], FLAGS[score_kernel] | QUERY_SPLIT[query_split] |
                 (QUERY_LAST_TOKEN if query == "last" else 0))
    h = ctypes.c_void_p()
    _check(LIB.litevlm_select_create(ctypes.byref(cfg), ctypes.byref(h)), None)
    return h.value


def destroy(handle: int) -> None:
    _check(LIB.litevlm_select_destroy(handle), handle)


def score(handle: int, batch: int, q_text, text_offsets_d, text_offsets_h, k_vis, seq_offsets_d, seq_offsets_h,
          q_scale: float, k_scale: float, scores, stream=None) -> None:
    rc = _FC.score(handle, batch, q_text, text_offsets_d, text_offsets_h, k_vis, seq_offsets_d, seq_offsets_h,
                   q_scale, k_scale, scores, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def score_full_keys(handle: int, batch: int, q_text, text_offsets_d, text_offsets_h, k_vis, seq_offsets_d,
                    seq_offsets_h, k_sys, sys_offsets_d, sys_offsets_h, k_text, q_scale: float, k_scale: float,
                    scores, stream=None) -> None:
    rc = _FC.score_full_keys(handle, batch, q_text, text_offsets_d, text_offsets_h, k_vis, seq_offsets_d,
                             seq_offsets_h, k_sys, sys_offsets_d, sys_offsets_h, k_text, q_scale, k_scale, scores,
                             _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def views(handle: int, batch: int, num_views: int, lexical, logits, tokens_per_view_h, w_lex: float, w_logit: float,
          threshold: float, min_views: int, view_mask, view_offsets, selected_views, seq_offsets,
          seq_offsets_h: Optional[np.ndarray] = None, stream=None) -> None:
    tpv = _host_i32(tokens_per_view_h)
    _check(LIB.litevlm_select_views(handle, batch, num_views, _ptr(lexical), _ptr(logits), _ptr(tpv), w_lex, w_logit,
                                    threshold, min_views, _ptr(view_mask), _ptr(view_offsets), _ptr(selected_views),
                                    _ptr(seq_offsets), _ptr(seq_offsets_h), _stream_ptr(stream)), handle)


def score_topk(handle: int, batch: int, q_text, text_offsets_d, text_offsets_h, k_vis, seq_offsets_d, seq_offsets_h,
               q_scale: float, k_scale: float, scores, keep_k_d, keep_k_h, keep_ratio: float, kept_idx,
               out_offsets_d, out_offsets_h, stream=None) -> None:
    rc = _FC.score_topk(handle, batch, q_text, text_offsets_d, text_offsets_h, k_vis, seq_offsets_d, seq_offsets_h,
                        q_scale, k_scale, scores, keep_k_d, keep_k_h, keep_ratio, kept_idx, out_offsets_d,
                        out_offsets_h, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def fold_norm(handle: int, out_features: int, hidden: int, w, gamma, w_folded, stream=None) -> None:
    _check(LIB.litevlm_select_fold_norm(handle, out_features, hidden, _ptr(w), _ptr(gamma), _ptr(w_folded),
                                        _stream_ptr(stream)), handle)


def rope_table(handle: int, max_positions: int, head_dim: int, rope_base: float, table, stream=None) -> None:
    _check(LIB.litevlm_select_rope_table(handle, max_positions, head_dim, rope_base, _ptr(table),
                                         _stream_ptr(stream)), handle)


def project(handle: int, rows: int, hidden: int, out_features: int, x, w_folded, bias, eps: float, head_dim: int,
            positions, table, max_positions: int, y, stream=None, out_scale: float = 0.0) -> None:
    rc = _FC.project(handle, rows, hidden, out_features, x, w_folded, bias, eps, head_dim, positions, table,
                     max_positions, out_scale, y, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def topk(handle: int, batch: int, scores, seq_offsets_d, seq_offsets_h, keep_k_d, keep_k_h, keep_ratio: float,
         kept_idx, out_offsets_d, out_offsets_h: Optional[np.ndarray] = None, stream=None) -> None:
    rc = _FC.topk(handle, batch, scores, seq_offsets_d, seq_offsets_h, keep_k_d, keep_k_h, keep_ratio, kept_idx,
                  out_offsets_d, out_offsets_h, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def compact(handle: int, total_kept: int, kept_idx, src_rows: int, srcs: Sequence, dsts: Sequence,
            row_bytes: Sequence[int], stream=None) -> None:
    n = len(srcs)
    if 1 <= n <= 8:
        rc = _FC.compact(handle, total_kept, kept_idx, src_rows, list(srcs), list(dsts), [int(r) for r in row_bytes],
                         _stream_ptr(stream))
    else:  # an error of the C call's
        src_arr = (ctypes.c_void_p * n)(*[_ptr(s) for s in srcs])
        dst_arr = (ctypes.c_void_p * n)(*[_ptr(d) for d in dsts])
        rb_arr = (ctypes.c_int64 * n)(*[int(r) for r in row_bytes])
        rc = LIB.litevlm_select_compact(handle, total_kept, _ptr(kept_idx), src_rows, n, src_arr, dst_arr, rb_arr,
                                        _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def splice(handle: int, batch: int, sys_rows, sys_offsets_d, sys_offsets_h, vis_rows, seq_offsets_d, seq_offsets_h,
           kept_idx, kept_offsets_d, kept_offsets_h, txt_rows, text_offsets_d, text_offsets_h, row_bytes: int,
           out_rows, out_offsets_d, position_ids, out_offsets_h: Optional[np.ndarray] = None, stream=None) -> None:
    rc = _FC.splice(handle, batch, sys_rows, sys_offsets_d, sys_offsets_h, vis_rows, seq_offsets_d, seq_offsets_h,
                    kept_idx, kept_offsets_d, kept_offsets_h, txt_rows, text_offsets_d, text_offsets_h,
                    int(row_bytes), out_rows, out_offsets_d, out_offsets_h, position_ids, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def cache_append(handle: int, batch: int, cache, table, table_width: int, seq_lens, k, k_row_stride: int, v,
                 v_row_stride: int, src_rows: int, row_idx, new_offsets_d, new_offsets_h, k_in_scale: float,
                 v_in_scale: float, weights, k_stored, v_stored, new_lens, stream=None, granted=None) -> None:
    """litevlm_select_cache_append, or with ``granted`` litevlm_select_cache_append_granted; cache: the address of a
    litevlm_cache_t (KVCache.struct)."""
    if granted is None:
        rc = _FC.cache_append(handle, batch, cache, table, table_width, seq_lens, k, k_row_stride, v, v_row_stride,
                              src_rows, row_idx, new_offsets_d, new_offsets_h, k_in_scale, v_in_scale, weights, k_stored,
                              v_stored, new_lens, _stream_ptr(stream))
    else:
        rc = _FC.cache_append_granted(handle, batch, cache, table, table_width, seq_lens, k, k_row_stride, v, v_row_stride,
                                      src_rows, row_idx, new_offsets_d, new_offsets_h, k_in_scale, v_in_scale, weights,
                                      k_stored, v_stored, granted, new_lens, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def cache_attend_workspace(handle: int, batch: int, q_offsets_h, max_len: int, weights: bool = True) -> int:
    """litevlm_select_cache_attend_workspace: bytes of the workspace of an attention call."""
    n = _FC.attend_bytes(handle, batch, q_offsets_h, max_len, weights)
    if n < 0:
        _check(-n, handle)
    return n


def cache_attend(handle: int, batch: int, cache, table, table_width: int, seq_lens, q, q_row_stride: int, q_offsets_d,
                 q_offsets_h, max_len: int, q_scale: float, weights_in, weights_out, out, workspace,
                 workspace_bytes: int, stream=None) -> None:
    rc = _FC.cache_attend(handle, batch, cache, table, table_width, seq_lens, q, q_row_stride, q_offsets_d, q_offsets_h,
                          max_len, q_scale, weights_in, weights_out, out, workspace, workspace_bytes,
                          _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def cache_evict(handle: int, batch: int, cache, table, table_width: int, seq_lens, max_len: int, budget: int, sink: int,
                recent: int, to_table, to_width: int, weights, kept_idx, new_lens, stream=None) -> None:
    rc = _FC.cache_evict(handle, batch, cache, table, table_width, seq_lens, max_len, budget, sink, recent, to_table,
                         to_width, weights, kept_idx, new_lens, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def cache_reserve(handle: int, batch: int, page_size: int, table, table_width: int, held, want, free_pages, num_pages: int,
                  state, new_offsets_d, new_offsets_h, granted, new_state, slots, stream=None) -> None:
    rc = _FC.cache_reserve(handle, batch, page_size, table, table_width, held, want, free_pages, num_pages, state,
                           new_offsets_d, new_offsets_h, granted, new_state, slots, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def cache_bounds(handle: int, batch: int, cache, bounds, table, table_width: int, seq_lens, new_offsets_d, new_offsets_h,
                 stream=None) -> None:
    """litevlm_select_cache_bounds; bounds: the address of a litevlm_key_bounds_t (KeyBounds.struct)."""
    rc = _FC.cache_bounds(handle, batch, cache, bounds, table, table_width, seq_lens, new_offsets_d, new_offsets_h,
                          _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def cache_pick_workspace(handle: int, batch: int, q_offsets_h, max_len: int, page_size: int, budget: int) -> int:
    """litevlm_select_cache_pick_workspace: bytes of the workspace of a selection of pages."""
    n = _FC.pick_bytes(handle, batch, q_offsets_h, max_len, page_size, budget)
    if n < 0:
        _check(-n, handle)
    return n


def cache_pick(handle: int, batch: int, bounds, table, table_width: int, seq_lens, q, q_row_stride: int, q_offsets_d,
               q_offsets_h, max_len: int, budget: int, sink: int, recent: int, picked, workspace, workspace_bytes: int,
               stream=None) -> None:
    rc = _FC.cache_pick(handle, batch, bounds, table, table_width, seq_lens, q, q_row_stride, q_offsets_d, q_offsets_h,
                        max_len, budget, sink, recent, picked, workspace, workspace_bytes, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def cache_attend_picked_workspace(handle: int, batch: int, q_offsets_h, page_size: int, table_width: int,
                                  budget: int) -> int:
    """litevlm_select_cache_attend_picked_workspace: bytes of the workspace of attention over picked pages."""
    n = _FC.picked_bytes(handle, batch, q_offsets_h, page_size, table_width, budget)
    if n < 0:
        _check(-n, handle)
    return n


def cache_attend_picked(handle: int, batch: int, cache, table, table_width: int, seq_lens, q, q_row_stride: int,
                        q_offsets_d, q_offsets_h, picked, budget: int, q_scale: float, out, workspace,
                        workspace_bytes: int, stream=None) -> None:
    rc = _FC.cache_attend_picked(handle, batch, cache, table, table_width, seq_lens, q, q_row_stride, q_offsets_d,
                                 q_offsets_h, picked, budget, q_scale, out, workspace, workspace_bytes,
                                 _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def verify(handle: int, batch: int, vocab: int, prob_bf16: int, draft_tokens, draft_offsets_d, draft_offsets_h,
           target_probs, draft_probs, u_accept, u_sample, accepted, tokens, stream=None) -> None:
    rc = _FC.verify(handle, batch, vocab, prob_bf16, draft_tokens, draft_offsets_d, draft_offsets_h, target_probs,
                    draft_probs, u_accept, u_sample, accepted, tokens, _stream_ptr(stream))
    if rc:
        _check(rc, handle)


def host_view(handle: int, host_ptr: int) -> int:
    """litevlm_select_host_view: the device address of pinned host memory."""
    out = ctypes.c_void_p()
    _check(LIB.litevlm_select_host_view(handle, host_ptr, ctypes.byref(out)), handle)
    return int(out.value)


def check_device(handle: int, stream=None) -> None:
    _check(LIB.litevlm_select_check_device(handle, _stream_ptr(stream)), handle)


def keep_offsets(seq_offsets_h, keep_k_h=None, keep_ratio: float = 0.0) -> np.ndarray:
    """litevlm_select_keep_offsets: prefix of the kept-token counts k_b (host only)."""
    so = _host_i32(seq_offsets_h)
    kk = _host_i32(keep_k_h)
    out = np.zeros(len(so), np.int32)
    _check(LIB.litevlm_select_keep_offsets(len(so) - 1, _ptr(so), _ptr(kk), keep_ratio, _ptr(out)), None)
    return out


def _keep_total(seq_offsets_h, keep_k_h, keep_ratio: float) -> int:
    """Kept tokens of a batch (the last of keep_offsets)."""
    total = _FC.keep_total(seq_offsets_h, keep_k_h, keep_ratio)
    if total < 0:
        _check(-total, None)
    return total


def set_wait_budget(handle: int, cycles: int) -> None:
    """litevlm_select_set_wait_budget: clock cycles each device-side wait may take (0: default)."""
    _check(LIB.litevlm_select_set_wait_budget(handle, int(cycles)), handle)


DEBUG_STALL_SCORE = 1
DEBUG_STALL_PROJECT = 4
DEBUG_STALL_ATTEND = 8
DEBUG_STALL_PICK = 16


def set_debug_flags(handle: int, flags: int) -> None:
    """litevlm_select_set_debug_flags: switches for tests of the failure path (0: off)."""
    _check(LIB.litevlm_select_set_debug_flags(handle, int(flags)), handle)


def score_noalloc(num_q_heads: int, num_kv_heads: int, head_dim: int, qk_dtype: str, batch: int, q_text,
                  text_offsets_d, text_offsets_h, k_vis, seq_offsets_d, seq_offsets_h, q_scale: float,
                  k_scale: float, scores, err_d, stream=None) -> None:
    """litevlm_select_score_noalloc: no handle, scratch in the library's static device arrays."""
    to_h, so_h = _host_i32(text_offsets_h), _host_i32(seq_offsets_h)
    _check(LIB.litevlm_select_score_noalloc(num_q_heads, num_kv_heads, head_dim, DTYPES[qk_dtype], batch,
                                            _ptr(q_text), _ptr(text_offsets_d), _ptr(to_h), _ptr(k_vis),
                                            _ptr(seq_offsets_d), _ptr(so_h), q_scale, k_scale, _ptr(scores),
                                            _ptr(err_d), _stream_ptr(stream)), None)


def score_plan(handle: int, batch: int, text_offsets_h, seq_offsets_h):
    """(kernel, cluster, tiles_per_cta, groups) litevlm_select_score would launch."""
    to_h, so_h = _host_i32(text_offsets_h), _host_i32(seq_offsets_h)
    out = np.zeros(4, np.int32)
    _check(LIB.litevlm_select_score_plan(handle, batch, _ptr(to_h), _ptr(so_h), _ptr(out)), handle)
    return tuple(int(v) for v in out)


# ----------------------------------------------------------------------------
# convenience object (allocates outputs with torch; still marshalling only)
# ----------------------------------------------------------------------------

def _refuse(message: str):
    raise LitevlmError(1, message)


def _want(name: str, t, dtype, shape, device: int):
    """A contiguous CUDA tensor of this type, shape (-1: any size) and device, or an error."""
    if _FC.fits(t, dtype, device, *shape):
        return t
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device.type != "cuda" or t.device.index != device:
        _refuse(f"{name} must be a {dtype} tensor on cuda:{device}")
    if t.dim() != len(shape) or any(w >= 0 and n != w for n, w in zip(t.shape, shape)):
        _refuse(f"{name} must have the shape {tuple('any' if w < 0 else w for w in shape)}, not {tuple(t.shape)}")
    _refuse(f"{name} must be contiguous")


def _row_stride(name: str, t, dtype, heads: int, d: int, device: int) -> int:
    """Elements from a row to the next of [rows, heads, d] rows, whose channels and heads lie side by side."""
    stride = _FC.row_stride(t, dtype, device, heads, d)
    if stride >= 0:
        return stride
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device.type != "cuda" or t.device.index != device:
        _refuse(f"{name} must be a {dtype} tensor on cuda:{device}")
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != d:
        _refuse(f"{name} must have the shape (any, {heads}, {d}), not {tuple(t.shape)}")
    _refuse(f"{name}'s heads and channels must lie side by side (only the row stride is free)")


def _bytes_of(t):
    """First address of a contiguous tensor's bytes and the one behind them."""
    return (0, 0) if t is None else (t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())


class KVCache:
    """The tensors of a 4-bit K/V cache (litevlm_cache_t), uint8 CUDA tensors: codes [pages, Hkv, page_size, d/2],
    scales [pages, Hkv, page_size, d/16]; weights: float32 [pages, page_size] or None. ``Selector.cache`` makes one.
    The calls are given the tensors' addresses and the scales once, so none of them can be assigned to; ``weights`` can."""

    def __setattr__(self, name, value):
        if name == "weights":
            if value is not None:
                import torch
                _want("weights", value, torch.float32, (self.num_pages, self.page_size), self.device)
            object.__setattr__(self, "weights_at", _bytes_of(value))
        elif "struct" in self.__dict__:
            _refuse(f"{name} of a KVCache is fixed: make another one")
        object.__setattr__(self, name, value)

    def __init__(self, k_codes, k_scales, v_codes, v_scales, k_scale: float = 1.0, v_scale: float = 1.0, weights=None):
        import torch
        if not isinstance(k_codes, torch.Tensor) or k_codes.dim() != 4 or k_codes.device.type != "cuda":
            _refuse("k_codes must be a CUDA tensor [pages, Hkv, page_size, d/2]")
        self.num_pages, self.heads, self.page_size = k_codes.shape[:3]
        self.head_dim = 2 * k_codes.shape[3]
        self.device = k_codes.device.index
        codes, scales = tuple(k_codes.shape), (*k_codes.shape[:3], self.head_dim // 16)
        for name, t, shape in (("k_codes", k_codes, codes), ("v_codes", v_codes, codes), ("k_scales", k_scales, scales),
                               ("v_scales", v_scales, scales)):
            _want(name, t, torch.uint8, shape, self.device)
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.k_scale, self.v_scale, self.weights = float(k_scale), float(v_scale), weights
        self._c = Cache(k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(),
                        self.num_pages, self.page_size, self.k_scale, self.v_scale)
        self.struct = ctypes.addressof(self._c)


class KeyBounds:
    """The ranges of a pool's keys (litevlm_key_bounds_t), int8 CUDA tensors: codes [pages, Hkv, 2, d] (largest, smallest),
    exps [pages, Hkv]. ``Selector.key_bounds`` makes one for a cache. Like a KVCache's its tensors are fixed."""

    def __setattr__(self, name, value):
        if "struct" in self.__dict__:
            _refuse(f"{name} of a KeyBounds is fixed: make another one")
        object.__setattr__(self, name, value)

    def __init__(self, codes, exps, page_size: int):
        import torch
        if not isinstance(codes, torch.Tensor) or codes.dim() != 4 or codes.device.type != "cuda":
            _refuse("codes must be a CUDA tensor [pages, Hkv, 2, d]")
        self.num_pages, self.heads, _, self.head_dim = codes.shape
        self.device, self.page_size = codes.device.index, int(page_size)
        _want("codes", codes, torch.int8, (self.num_pages, self.heads, 2, self.head_dim), self.device)
        _want("exps", exps, torch.int8, (self.num_pages, self.heads), self.device)
        self.codes, self.exps = codes, exps
        self.at = (_bytes_of(codes), _bytes_of(exps))
        self._c = Bounds(codes.data_ptr(), exps.data_ptr(), self.num_pages, self.page_size)
        self.struct = ctypes.addressof(self._c)


class _NoContext:
    def __enter__(self):
        return None

    def __exit__(self, *a):
        return False


_HERE = _NoContext()


def _allocate_on(stream, device: int):
    """Where a call has a stream of its own, its buffers belong to that stream (the allocator then gives their memory
    to nobody else before the call's work has run)."""
    if stream is None:
        return _HERE
    import torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def _stream_on(stream, device: int) -> int:
    """The raw stream of a call: the one given, or the current one of the tensors' device."""
    if stream is not None:
        return _stream_ptr(stream)
    import torch
    return torch._C._cuda_getCurrentRawStream(device)


class Selector:
    """Owns one handle. Tensors are torch CUDA tensors laid out as in the C header."""

    def __init__(self, max_batch: int, max_total_visual: int, max_total_text: int, num_q_heads: int,
                 num_kv_heads: int, head_dim: int, qk_dtype: str = "bf16", score_kernel: str = "auto",
                 query: str = "all", query_split: str = "whole"):
        self.handle = create(max_batch, max_total_visual, max_total_text, num_q_heads, num_kv_heads, head_dim,
                             qk_dtype, score_kernel, query, query_split)
        self.qk_dtype = qk_dtype
        self.heads, self.kv_heads, self.head_dim = num_q_heads, num_kv_heads, head_dim
        import torch
        self.device = torch.cuda.current_device()  # the one that create() took
        self._space = None  # the stream and the workspace of the last cache_attend

    def close(self) -> None:
        self._space = None
        if self.handle:
            destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def score(self, q, text_offsets, k, seq_offsets, q_scale=1.0, k_scale=1.0, out=None, text_offsets_h=None,
              seq_offsets_h=None, stream=None):
        import torch
        so_h = _host_i32(seq_offsets if seq_offsets_h is None else seq_offsets_h)
        to_h = _host_i32(text_offsets if text_offsets_h is None else text_offsets_h)
        if out is None:
            out = torch.empty(int(so_h[-1]), dtype=torch.float32, device=k.device)
        score(self.handle, len(so_h) - 1, q, text_offsets, to_h, k, seq_offsets, so_h, q_scale, k_scale, out,
              stream)
        return out

    def score_full_keys(self, q, text_offsets, k, seq_offsets, k_sys, sys_offsets, k_text, q_scale=1.0,
                        k_scale=1.0, out=None, text_offsets_h=None, seq_offsets_h=None, sys_offsets_h=None,
                        stream=None):
        """Scores with the softmax over [system; visual; causal text] keys."""
        import torch
        so_h = _host_i32(seq_offsets if seq_offsets_h is None else seq_offsets_h)
        to_h = _host_i32(text_offsets if text_offsets_h is None else text_offsets_h)
        yo_h = _host_i32(sys_offsets if sys_offsets_h is None else sys_offsets_h)
        if out is None:
            out = torch.empty(int(so_h[-1]), dtype=torch.float32, device=k.device)
        score_full_keys(self.handle, len(so_h) - 1, q, text_offsets, to_h, k, seq_offsets, so_h, k_sys, sys_offsets,
                        yo_h, k_text, q_scale, k_scale, out, stream)
        return out

    def select_views(self, lexical, logits, tokens_per_view, w_lex: float, w_logit: float, threshold: float,
                     min_views: int = 0, stream=None):
        """Patch-selection gating on float32 CUDA tensors [B, V]. Returns
        (view_mask, view_offsets, selected_views, seq_offsets device tensors,
        seq_offsets host numpy; the call synchronises to fill the latter)."""
        import torch
        batch, nv = lexical.shape
        dev = lexical.device
        mask = torch.empty((max(batch, 1), nv), dtype=torch.uint8, device=dev)
        vo = torch.empty(batch + 1, dtype=torch.int32, device=dev)
        sv = torch.empty(max(batch * nv, 1), dtype=torch.int32, device=dev)
        so = torch.empty(batch + 1, dtype=torch.int32, device=dev)
        so_h = np.zeros(batch + 1, np.int32)
        views(self.handle, batch, nv, lexical, logits, tokens_per_view, w_lex, w_logit, threshold, min_views, mask,
              vo, sv, so, so_h, stream)
        return mask[:batch], vo, sv, so, so_h

    def score_topk(self, q, text_offsets, k, seq_offsets, q_scale=1.0, k_scale=1.0, keep_k=None,
                   keep_ratio: float = 0.0, text_offsets_h=None, seq_offsets_h=None, stream=None, out=None,
                   kept_idx=None, out_offsets=None):
        """Scores and top-k in one call. Returns (scores, kept_idx, out_offsets
        device, out_offsets host numpy); out / kept_idx / out_offsets are
        optional caller buffers."""
        import torch
        so_h = _host_i32(seq_offsets if seq_offsets_h is None else seq_offsets_h)
        to_h = _host_i32(text_offsets if text_offsets_h is None else text_offsets_h)
        batch = len(so_h) - 1
        kk_h = _host_i32(keep_k)
        kk_d = None
        if kk_h is not None:
            kk_d = keep_k if isinstance(keep_k, torch.Tensor) and keep_k.is_cuda else \
                torch.from_numpy(kk_h).to(k.device)
        total, n, dev = _keep_total(so_h, kk_h, keep_ratio), int(so_h[-1]), k.device
        scores = out if out is not None else torch.empty(max(1, n), dtype=torch.float32, device=dev)
        kept = kept_idx if kept_idx is not None else torch.empty(max(total, 1), dtype=torch.int32, device=dev)
        off_d = out_offsets if out_offsets is not None else torch.empty(batch + 1, dtype=torch.int32, device=dev)
        off_h = np.zeros(batch + 1, np.int32)
        score_topk(self.handle, batch, q, text_offsets, to_h, k, seq_offsets, so_h, q_scale, k_scale, scores, kk_d,
                   kk_h, keep_ratio, kept, off_d, off_h, stream)
        self._keep_alive = kk_d
        # (a buffer made here already has its length, unless that is 0)
        return (scores if out is None and n else scores[:n], kept if kept_idx is None and total else kept[:total],
                off_d, off_h)

    def fold_norm(self, w, gamma, stream=None):
        """bf16 W * gamma (per input column) for project()."""
        import torch
        out = torch.empty_like(w)
        fold_norm(self.handle, w.shape[0], w.shape[1], w, gamma, out, stream)
        return out

    def rope_table(self, max_positions: int, head_dim: int, rope_base: float, device="cuda", stream=None):
        import torch
        t = torch.empty((max_positions, head_dim // 2, 2), dtype=torch.float32, device=device)
        rope_table(self.handle, max_positions, head_dim, rope_base, t, stream)
        return t

    def project(self, x, w_folded, bias=None, eps: float = 1e-6, head_dim: int = 0, positions=None, table=None,
                out=None, stream=None, out_scale: float = 0.0):
        """y = RoPE(RMS-scale(x) . w_folded^T + bias): bf16 [rows, out_features],
        or uint8 e4m3 codes of y / out_scale when out_scale > 0."""
        import torch
        rows, hidden = x.shape
        out_f = w_folded.shape[0]
        if out is None:
            out = torch.empty((rows, out_f), dtype=torch.uint8 if out_scale > 0 else torch.bfloat16,
                              device=x.device)
        project(self.handle, rows, hidden, out_f, x, w_folded, bias, eps, head_dim, positions, table,
                0 if table is None else table.shape[0], out, stream, out_scale)
        return out

    def topk(self, scores, seq_offsets, keep_k=None, keep_ratio: float = 0.0, seq_offsets_h=None, kept_idx=None,
             out_offsets=None, stream=None):
        """Returns (kept_idx, out_offsets device tensor, out_offsets host numpy)."""
        import torch
        so_h = _host_i32(seq_offsets if seq_offsets_h is None else seq_offsets_h)
        batch = len(so_h) - 1
        kk_h = _host_i32(keep_k)
        kk_d = None
        if kk_h is not None:
            kk_d = keep_k if isinstance(keep_k, torch.Tensor) and keep_k.is_cuda else \
                torch.from_numpy(kk_h).to(scores.device)
        off_h = np.zeros(batch + 1, dtype=np.int32)
        total = _keep_total(so_h, kk_h, keep_ratio)
        made = kept_idx is None and total > 0
        if kept_idx is None:
            kept_idx = torch.empty(max(total, 1), dtype=torch.int32, device=scores.device)
        if out_offsets is None:
            out_offsets = torch.empty(batch + 1, dtype=torch.int32, device=scores.device)
        topk(self.handle, batch, scores, seq_offsets, so_h, kk_d, kk_h, keep_ratio, kept_idx, out_offsets, off_h,
             stream)
        self._keep_alive = kk_d
        return kept_idx if made else kept_idx[:total], out_offsets, off_h

    def compact(self, kept_idx, total_kept: int, srcs: Sequence, dsts: Optional[List] = None, stream=None):
        """Gathers the kept rows of each source into the device. A source in
        pinned host memory is read through its device view, so only its kept
        rows cross the host link."""
        import torch
        rows = [s.shape[0] for s in srcs]
        if dsts is None:
            dev, n = kept_idx.device, max(total_kept, 0)
            dsts = [torch.empty((n, *s.shape[1:]), dtype=s.dtype, device=dev) for s in srcs]
        rb = [s.nbytes // r if r else 1 for s, r in zip(srcs, rows)]
        src_ptrs = [s if s.is_cuda else self.host_view(s) for s in srcs]
        compact(self.handle, total_kept, kept_idx, min(rows) if rows else 0, src_ptrs, dsts, rb, stream)
        return dsts

    def host_view(self, t) -> int:
        """Device address of a pinned host tensor (or host pointer)."""
        return host_view(self.handle, _ptr(t))

    def splice(self, sys_rows, sys_offsets, vis_rows, seq_offsets, kept_idx, kept_offsets, txt_rows, text_offsets,
               stream=None):
        """[system; kept visual; text] rows per request and their original
        position ids. Rows are 2-D torch CUDA tensors with equal row sizes;
        offsets are int32 CUDA tensors. Returns (rows, out_offsets, out_offsets
        host numpy, position_ids)."""
        import torch
        so, vo, ko, to = (_host_i32(a) for a in (sys_offsets, seq_offsets, kept_offsets, text_offsets))
        batch = len(so) - 1
        total = int(so[-1] + ko[-1] + to[-1])
        ref = next(r for r in (sys_rows, vis_rows, txt_rows) if r is not None)
        rb = ref[0].numel() * ref.element_size() if ref.shape[0] else ref.element_size() * int(np.prod(ref.shape[1:]))
        out = torch.empty((max(total, 1),) + tuple(ref.shape[1:]), dtype=ref.dtype, device=ref.device)
        pos = torch.empty(max(total, 1), dtype=torch.int32, device=ref.device)
        off_d = torch.empty(batch + 1, dtype=torch.int32, device=ref.device)
        off_h = np.zeros(batch + 1, np.int32)
        splice(self.handle, batch, sys_rows, sys_offsets, so, vis_rows, seq_offsets, vo, kept_idx, kept_offsets, ko,
               txt_rows, text_offsets, to, rb, out, off_d, pos, off_h, stream)
        return out[:total], off_d, off_h, pos[:total]

    # ---- the 4-bit K/V cache

    def _cache_call(self, cache, table, seq_lens, batch: int, kind=KVCache):
        import torch
        if not isinstance(cache, kind):
            _refuse(f"{'cache' if kind is KVCache else 'bounds'} must be a {kind.__name__}")
        if cache.device != self.device:
            _refuse(f"the cache is on cuda:{cache.device}, the handle on cuda:{self.device}")
        if cache.heads != self.kv_heads or cache.head_dim != self.head_dim:
            _refuse(f"the cache has {cache.heads} heads of {cache.head_dim}, the handle {self.kv_heads} of "
                    f"{self.head_dim}")
        _want("table", table, torch.int32, (batch, -1), cache.device)
        _want("seq_lens", seq_lens, torch.int32, (batch,), cache.device)
        return cache.device

    def _workspace(self, need: int, stream, device):
        """The handle's own workspace for calls on one stream after another (an earlier stream's goes back to the
        allocator); a call that is captured, or that has a stream of its own, gets one that nothing else uses."""
        import torch
        if stream is not None or torch._C._cuda_isCurrentStreamCapturing():
            return torch.empty(need, dtype=torch.uint8, device=device)
        now = torch._C._cuda_getCurrentRawStream(device.index)
        if self._space is None or self._space[0] != now or self._space[1].shape[0] < need:
            self._space = None
            self._space = (now, torch.empty(need, dtype=torch.uint8, device=device))
        return self._space[1]

    def _element(self):
        import torch
        return torch.uint8 if self.qk_dtype == "e4m3" else torch.bfloat16

    def cache(self, num_pages: int, page_size: int, k_scale: float = 1.0, v_scale: float = 1.0, weights: bool = True,
              device=None) -> KVCache:
        """An empty cache of the handle's head sizes (on the handle's device)."""
        import torch
        device = self.device if device is None else device
        shape = (num_pages, self.kv_heads, page_size)
        c = [torch.zeros((*shape, self.head_dim // n), dtype=torch.uint8, device=device) for n in (2, 16, 2, 16)]
        w = torch.zeros((num_pages, page_size), dtype=torch.float32, device=device) if weights else None
        return KVCache(*c, k_scale=k_scale, v_scale=v_scale, weights=w)

    def cache_append(self, cache: KVCache, table, seq_lens, k, v, offsets, rows=None, k_in_scale: float = 1.0,
                     v_in_scale: float = 1.0, offsets_h=None, stored: bool = False, new_lens=None, stream=None,
                     granted=None):
        """Quantises rows into the cache: token t of request b, row offsets[b] + t of k and v [rows, Hkv, d] (or row
        rows[offsets[b] + t]), to position seq_lens[b] + t of the request's pages; its weight becomes 0. With ``granted``
        (what ``cache_reserve`` returned) the tokens behind it are skipped: a refused request stays as it was. Returns
        the new lengths, and with ``stored`` also the K and V values that the cache now holds for the rows (bf16)."""
        import torch
        off_h = _host_i32(offsets if offsets_h is None else offsets_h)
        batch, total = len(off_h) - 1, int(off_h[-1])
        dev = self._cache_call(cache, table, seq_lens, batch)
        _want("offsets", offsets, torch.int32, (batch + 1,), dev)
        kind = self._element()
        k_stride = _row_stride("k", k, kind, self.kv_heads, self.head_dim, dev)
        v_stride = _row_stride("v", v, kind, self.kv_heads, self.head_dim, dev)
        if v.shape[0] != k.shape[0]:
            _refuse("k and v must have the same number of rows")
        if rows is not None:
            _want("rows", rows, torch.int32, (total,), dev)
        if granted is not None:
            _want("granted", granted, torch.int32, (batch,), dev)
        with _allocate_on(stream, dev):
            if new_lens is None:
                new_lens = torch.empty_like(seq_lens)
            else:
                _want("new_lens", new_lens, torch.int32, (batch,), dev)
            out = [torch.empty((total, self.kv_heads, self.head_dim), dtype=torch.bfloat16, device=k.device)
                   for _ in "kv"] if stored else (None, None)
        cache_append(self.handle, batch, cache.struct, table, table.shape[1], seq_lens, k, k_stride, v, v_stride,
                     k.shape[0], rows, offsets, off_h, k_in_scale, v_in_scale, cache.weights, out[0], out[1], new_lens,
                     _stream_on(stream, dev), granted)
        return (new_lens, *out) if stored else new_lens

    def cache_attend(self, cache: KVCache, table, seq_lens, q, offsets, max_len: int, q_scale: float = 1.0,
                     accumulate: bool = False, weights_out=None, offsets_h=None, out=None, workspace=None, stream=None):
        """Attention of each request's last tokens (queries [sum T, Hq, d], offsets the prefix of T) over its cache.
        ``accumulate`` adds every cached token's attention weight (mean over heads, summed over queries) to
        cache.weights in place; ``weights_out`` takes the sums instead and leaves cache.weights as it is. Returns the
        bf16 outputs [sum T, Hq, d]. ``workspace``: a uint8 tensor of at least ``cache_attend_workspace`` bytes that no
        other call in flight uses (made for the call when not given)."""
        import torch
        off_h = _host_i32(offsets if offsets_h is None else offsets_h)
        batch, total = len(off_h) - 1, int(off_h[-1])
        dev = self._cache_call(cache, table, seq_lens, batch)
        _want("offsets", offsets, torch.int32, (batch + 1,), dev)
        stride = _row_stride("q", q, self._element(), self.heads, self.head_dim, dev)
        if q.shape[0] != total:
            _refuse(f"q has {q.shape[0]} rows, the offsets {total}")
        w_in = w_out = None
        if weights_out is not None or accumulate:
            if cache.weights is None:
                _refuse("the cache has no weights")
            w_in = w_out = cache.weights
            if weights_out is not None:
                w_out = _want("weights_out", weights_out, torch.float32, (cache.num_pages, cache.page_size), dev)
        need = cache_attend_workspace(self.handle, batch, off_h, max_len, w_out is not None)
        with _allocate_on(stream, dev):
            if out is None:
                out = torch.empty((total, self.heads, self.head_dim), dtype=torch.bfloat16, device=q.device)
            else:
                _want("out", out, torch.bfloat16, (total, self.heads, self.head_dim), dev)
            if workspace is None:
                workspace = self._workspace(need, stream, q.device)
            else:
                _want("workspace", workspace, torch.uint8, (-1,), dev)
        cache_attend(self.handle, batch, cache.struct, table, table.shape[1], seq_lens, q, stride, offsets, off_h,
                     max_len, q_scale, w_in, w_out, out, workspace, workspace.shape[0], _stream_on(stream, dev))
        return out

    def cache_evict(self, cache: KVCache, table, seq_lens, max_len: int, budget: int, sink: int = 0, recent: int = 0,
                    to_table=None, new_lens=None, kept_idx=None, stream=None):
        """Cuts every request back to ``budget`` tokens: its first ``sink``, its last ``recent`` and the others of the
        largest cache.weights stay, in order, at the front of the request's pages (or of the pages of to_table).
        Returns (kept positions int32 [batch, budget], -1 behind the last; new lengths)."""
        import torch
        batch = seq_lens.shape[0] if isinstance(seq_lens, torch.Tensor) and seq_lens.dim() == 1 else -1
        dev = self._cache_call(cache, table, seq_lens, batch)
        if cache.weights is None:
            _refuse("the cache has no weights")
        if to_table is not None:
            _want("to_table", to_table, torch.int32, (batch, -1), dev)
        with _allocate_on(stream, dev):
            if new_lens is None:
                new_lens = torch.empty_like(seq_lens)
            else:
                _want("new_lens", new_lens, torch.int32, (batch,), dev)
            if kept_idx is None:
                kept_idx = torch.empty((batch, max(budget, 0)), dtype=torch.int32, device=seq_lens.device)
            else:
                _want("kept_idx", kept_idx, torch.int32, (batch, max(budget, 0)), dev)
        cache_evict(self.handle, batch, cache.struct, table, table.shape[1], seq_lens, max_len, budget, sink, recent,
                    to_table, 0 if to_table is None else to_table.shape[1], cache.weights, kept_idx, new_lens,
                    _stream_on(stream, dev))
        return kept_idx, new_lens

    # ---- its pages: who has them, and attention over some of them. Their tensors are checked in one call where all fit
    # (the single checks then say what does not): of a decoding step's calls the host's part is the longer one.

    def _pages_fit(self, pages, kind, dev: int) -> bool:
        return type(pages) is kind and pages.device == dev and pages.heads == self.kv_heads and \
            pages.head_dim == self.head_dim

    def cache_reserve(self, table, held, want, free, state, page_size: int, offsets, offsets_h=None, granted=None,
                      new_state=None, slots=None, stream=None):
        """Gives pages to requests that hold ``held`` tokens and are to hold ``want``, or takes them back: from and to the
        ring ``free`` (int32, as long as the pool), whose head and count are ``state``; ``table`` and ``free`` are updated in
        place. ``offsets``: the prefix of the new tokens among each request's want. Returns (granted: want, or held where the
        ring had too few pages; the ring's new state; slots int64 of the new tokens, -1 for those that were not granted)."""
        import torch
        off_h = _host_i32(offsets if offsets_h is None else offsets_h)
        batch, total, dev, i32 = len(off_h) - 1, int(off_h[-1]), self.device, torch.int32
        if not _FC.all_fit(dev, i32, table, 2, batch, -1, held, 1, batch, want, 1, batch, free, 1, -1, state, 1, 2, offsets, 1,
                           batch + 1):
            _want("table", table, i32, (batch, -1), dev)
            _want("held", held, i32, (batch,), dev)
            _want("want", want, i32, (batch,), dev)
            _want("free", free, i32, (-1,), dev)
            _want("state", state, i32, (2,), dev)
            _want("offsets", offsets, i32, (batch + 1,), dev)
        if granted is None and new_state is None and slots is None and stream is None:
            granted, new_state = torch.empty_like(held), torch.empty_like(state)
            slots = torch.empty(total, dtype=torch.int64, device=held.device)
        else:
            with _allocate_on(stream, dev):
                granted = torch.empty_like(held) if granted is None else _want("granted", granted, i32, (batch,), dev)
                new_state = torch.empty_like(state) if new_state is None else _want("new_state", new_state, i32, (2,), dev)
                slots = torch.empty(total, dtype=torch.int64, device=held.device) if slots is None else \
                    _want("slots", slots, torch.int64, (total,), dev)
        rc = _FC.cache_reserve(self.handle, batch, page_size, table, table.shape[1], held, want, free, free.shape[0], state,
                               offsets, off_h, granted, new_state, slots, _stream_on(stream, dev))
        if rc:
            _check(rc, self.handle)
        return granted, new_state, slots

    def key_bounds(self, cache: KVCache) -> KeyBounds:
        """Empty ranges for a cache's pages (``cache_bounds`` fills them)."""
        import torch
        device = cache.k_codes.device
        return KeyBounds(torch.zeros((cache.num_pages, cache.heads, 2, cache.head_dim), dtype=torch.int8, device=device),
                         torch.zeros((cache.num_pages, cache.heads), dtype=torch.int8, device=device), cache.page_size)

    def cache_bounds(self, cache: KVCache, bounds: KeyBounds, table, seq_lens, offsets, offsets_h=None, stream=None):
        """Renews the ranges of the pages that hold each request's last tokens (``offsets``: the prefix of their numbers;
        ``seq_lens`` with them), from all tokens of these pages."""
        import torch
        off_h = _host_i32(offsets if offsets_h is None else offsets_h)
        batch, dev = len(off_h) - 1, self.device
        if not (self._pages_fit(cache, KVCache, dev) and self._pages_fit(bounds, KeyBounds, dev) and
                _FC.all_fit(dev, torch.int32, table, 2, batch, -1, seq_lens, 1, batch, offsets, 1, batch + 1)):
            self._cache_call(cache, table, seq_lens, batch)
            self._cache_call(bounds, table, seq_lens, batch, KeyBounds)
            _want("offsets", offsets, torch.int32, (batch + 1,), dev)
        first, end = cache.weights_at  # (the C call does not know them)
        (a0, b0), (a1, b1) = bounds.at
        if a0 < end and first < b0 or a1 < end and first < b1:
            _refuse("the ranges must not overlap the cache's weights")
        rc = _FC.cache_bounds(self.handle, batch, cache.struct, bounds.struct, table, table.shape[1], seq_lens, offsets, off_h,
                              _stream_on(stream, dev))
        if rc:
            _check(rc, self.handle)
        return bounds

    def _queries(self, pages, kind, table, seq_lens, q, offsets, batch: int, total: int, dev: int) -> int:
        """The row stride of q, the other tensors of a call on cached pages checked."""
        import torch
        stride = _FC.row_stride(q, self._element(), dev, self.heads, self.head_dim)
        if stride < 0 or q.shape[0] != total or not self._pages_fit(pages, kind, dev) or \
                not _FC.all_fit(dev, torch.int32, table, 2, batch, -1, seq_lens, 1, batch, offsets, 1, batch + 1):
            self._cache_call(pages, table, seq_lens, batch, kind)
            _want("offsets", offsets, torch.int32, (batch + 1,), dev)
            stride = _row_stride("q", q, self._element(), self.heads, self.head_dim, dev)
            if q.shape[0] != total:
                _refuse(f"q has {q.shape[0]} rows, the offsets {total}")
        return stride

    def cache_pick(self, bounds: KeyBounds, table, seq_lens, q, offsets, max_len: int, budget: int, sink: int = 0,
                   recent: int = 0, offsets_h=None, picked=None, workspace=None, stream=None):
        """The ``budget`` pages that each query [sum T, Hq, d] attends to, for each key head: the first ``sink``, the last
        ``recent`` up to its own position, and those whose ranges have the largest product with it. Returns int32
        [sum T, Hkv, budget]: pages of the request, ascending, -1 behind the last. ``workspace``: a uint8 tensor of at least
        ``cache_pick_workspace`` bytes (4 for every query, key head and page of ``max_len``, whatever the lengths are) that
        no other call in flight uses; without one the handle keeps its own, of the largest call so far."""
        import torch
        off_h = _host_i32(offsets if offsets_h is None else offsets_h)
        batch, total, dev = len(off_h) - 1, int(off_h[-1]), self.device
        stride = self._queries(bounds, KeyBounds, table, seq_lens, q, offsets, batch, total, dev)
        need = _FC.pick_bytes(self.handle, batch, off_h, max_len, bounds.page_size, budget)
        if need < 0:
            _check(-need, self.handle)
        if picked is None and workspace is None and stream is None:
            picked = torch.empty((total, self.kv_heads, budget), dtype=torch.int32, device=q.device)
            if need:
                workspace = self._workspace(need, None, q.device)
        else:
            with _allocate_on(stream, dev):
                picked = torch.empty((total, self.kv_heads, budget), dtype=torch.int32, device=q.device) if picked is None \
                    else _want("picked", picked, torch.int32, (total, self.kv_heads, budget), dev)
                if workspace is not None:
                    need = _want("workspace", workspace, torch.uint8, (-1,), dev).shape[0]
                elif need:
                    workspace = self._workspace(need, stream, q.device)
        rc = _FC.cache_pick(self.handle, batch, bounds.struct, table, table.shape[1], seq_lens, q, stride, offsets, off_h,
                            max_len, budget, sink, recent, picked, workspace, need, _stream_on(stream, dev))
        if rc:
            _check(rc, self.handle)
        return picked

    def cache_attend_picked(self, cache: KVCache, table, seq_lens, q, offsets, picked, q_scale: float = 1.0,
                            offsets_h=None, out=None, workspace=None, stream=None):
        """``cache_attend`` over the pages that ``picked`` (int32 [sum T, Hkv, budget]) names for each query and key head;
        entries that are no page that the query sees are skipped. Returns the bf16 outputs [sum T, Hq, d]."""
        import torch
        off_h = _host_i32(offsets if offsets_h is None else offsets_h)
        batch, total, dev = len(off_h) - 1, int(off_h[-1]), self.device
        stride = self._queries(cache, KVCache, table, seq_lens, q, offsets, batch, total, dev)
        _want("picked", picked, torch.int32, (total, self.kv_heads, -1), dev)
        budget, shape = picked.shape[2], (total, self.heads, self.head_dim)
        need = _FC.picked_bytes(self.handle, batch, off_h, cache.page_size, table.shape[1], budget)
        if need < 0:
            _check(-need, self.handle)
        if out is None and workspace is None and stream is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
            if need:
                workspace = self._workspace(need, None, q.device)
        else:
            with _allocate_on(stream, dev):
                out = torch.empty(shape, dtype=torch.bfloat16, device=q.device) if out is None \
                    else _want("out", out, torch.bfloat16, shape, dev)
                if workspace is not None:
                    need = _want("workspace", workspace, torch.uint8, (-1,), dev).shape[0]
                elif need:
                    workspace = self._workspace(need, stream, q.device)
        rc = _FC.cache_attend_picked(self.handle, batch, cache.struct, table, table.shape[1], seq_lens, q, stride, offsets,
                                     off_h, picked, budget, q_scale, out, workspace, need, _stream_on(stream, dev))
        if rc:
            _check(rc, self.handle)
        return out

    def verify(self, draft_tokens, target_probs, u_accept, u_sample, offsets, draft_probs=None, offsets_h=None,
               accepted=None, tokens=None, stream=None):
        """Verifies drafted tokens (int32 [sum T]) against the target's probabilities [sum T + B, vocab] (float32 or
        bf16; draft_probs [sum T, vocab] likewise, None: the drafts were certain). Returns (accepted drafts of every
        request, tokens [sum T + B]: request b's accepted drafts, the sampled token, then -1, from offsets[b] + b)."""
        import torch
        off_h = _host_i32(offsets if offsets_h is None else offsets_h)
        batch, total = len(off_h) - 1, int(off_h[-1])
        if not isinstance(target_probs, torch.Tensor) or target_probs.device.type != "cuda" or \
                target_probs.dim() != 2 or target_probs.dtype not in (torch.float32, torch.bfloat16):
            _refuse("target_probs must be a float32 or bf16 CUDA tensor [sum T + batch, vocab]")
        dev, kind, vocab = target_probs.device.index, target_probs.dtype, target_probs.shape[1]
        if dev != self.device:
            _refuse(f"target_probs is on cuda:{dev}, the handle on cuda:{self.device}")
        _want("target_probs", target_probs, kind, (total + batch, -1), dev)
        _want("draft_tokens", draft_tokens, torch.int32, (total,), dev)
        _want("u_accept", u_accept, torch.float32, (total,), dev)
        _want("u_sample", u_sample, torch.float32, (batch,), dev)
        _want("offsets", offsets, torch.int32, (batch + 1,), dev)
        if draft_probs is not None:
            _want("draft_probs", draft_probs, kind, (total, vocab), dev)
        with _allocate_on(stream, dev):
            if accepted is None:
                accepted = torch.empty(batch, dtype=torch.int32, device=target_probs.device)
            else:
                _want("accepted", accepted, torch.int32, (batch,), dev)
            if tokens is None:
                tokens = torch.empty(total + batch, dtype=torch.int32, device=target_probs.device)
            else:
                _want("tokens", tokens, torch.int32, (total + batch,), dev)
        verify(self.handle, batch, vocab, int(kind == torch.bfloat16), draft_tokens, offsets, off_h, target_probs,
               draft_probs, u_accept, u_sample, accepted, tokens, _stream_on(stream, dev))
        return accepted, tokens

    def check_device(self, stream=None) -> None:
        check_device(self.handle, stream)

    def set_wait_budget(self, cycles: int) -> None:
        set_wait_budget(self.handle, cycles)

    def set_debug_flags(self, flags: int) -> None:
        set_debug_flags(self.handle, flags)

    def score_plan(self, text_offsets_h, seq_offsets_h):
        so = _host_i32(seq_offsets_h)
        return score_plan(self.handle, len(so) - 1, text_offsets_h, so)
