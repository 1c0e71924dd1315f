"""ctypes binding of libactkv.so: the same names as the C ABI, argument marshalling only.

Tensors are torch CUDA tensors (torch is used for device memory and streams, nothing else);
each wrapper checks dtype / device / contiguity, passes raw pointers and raises `ActKVError`
on a non-zero return code.  There is no fallback: a missing or unloadable library is an error.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libactkv.so")

OK, E_INVALID, E_WORKSPACE, E_CUDA, E_BADPAGE, E_NOFREE, E_BADINDEX, E_TIMEOUT = 0, -1, -2, -3, -4, -5, -6, -7
STALL_ANSWER = 0x7fffffff
E_TOOBIG = -8
ERROR_NAMES = {E_INVALID: "ACTKV_E_INVALID", E_WORKSPACE: "ACTKV_E_WORKSPACE", E_CUDA: "ACTKV_E_CUDA",
               E_BADPAGE: "ACTKV_E_BADPAGE", E_NOFREE: "ACTKV_E_NOFREE", E_BADINDEX: "ACTKV_E_BADINDEX",
               E_TIMEOUT: "ACTKV_E_TIMEOUT", E_TOOBIG: "ACTKV_E_TOOBIG"}

EXPORTS = ["actkv_budget_workspace_bytes", "actkv_budget", "actkv_score_workspace_bytes", "actkv_score",
           "actkv_score_lse", "actkv_score_accumulate",
           "actkv_keep_indptr", "actkv_select_workspace_bytes", "actkv_select",
           "actkv_compact_workspace_bytes", "actkv_compact", "actkv_compact_noalloc",
           "actkv_compact_noalloc_max_bytes", "actkv_step_host", "actkv_step_device", "actkv_keepscore", "actkv_gather_f32",
           "actkv_compact_inplace", "actkv_score_path", "actkv_debug_inject_stall", "actkv_score_sliding", "actkv_keepscore_select",
           "actkv_compact_deferred_workspace_bytes", "actkv_compact_begin", "actkv_compact_end", "actkv_score_overlap", "actkv_compact_stats",
           "actkv_compact_inplace_deferred_workspace_bytes", "actkv_compact_inplace_begin", "actkv_compact_inplace_end",
           "actkv_attend_workspace_bytes", "actkv_attend", "actkv_append", "actkv_resize", "actkv_copy", "actkv_logprob",
           "actkv_reposition", "actkv_penalize", "actkv_sample", "actkv_version"]


class ActKVError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} returned {code} ({ERROR_NAMES.get(code, 'unknown')})")
        self.code = code


class PoolDesc(C.Structure):
    _fields_ = [("base", C.c_void_p), ("n_layers", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("stride_layer", C.c_int64),
                ("stride_kv", C.c_int64), ("stride_page", C.c_int64), ("stride_slot", C.c_int64),
                ("stride_head", C.c_int64)]


class TablesDesc(C.Structure):
    _fields_ = [("n_req", C.c_int32), ("max_pages", C.c_int32), ("page_table", C.c_void_p),
                ("seq_len", C.c_void_p), ("free_list", C.c_void_p), ("free_count", C.c_void_p)]


class BudgetParams(C.Structure):
    _fields_ = [("k", C.c_int32), ("w", C.c_int32), ("s", C.c_int32), ("b_percent", C.c_double),
                ("scale_up", C.c_double), ("B_upper", C.c_int32), ("clamp_lo_ppm", C.c_int32),
                ("clamp_hi_ppm", C.c_int32)]

    @classmethod
    def paper_defaults(cls, clamp_lo_ppm: int = 0, clamp_hi_ppm: int = 0):
        return cls(20, 64, 8, 10.0, 1.75, 30000, clamp_lo_ppm, clamp_hi_ppm)


class TieReport(C.Structure):
    _fields_ = [("threshold", C.c_float), ("n_equal_kept", C.c_int32), ("n_equal_total", C.c_int32),
                ("n_keep", C.c_int32)]


class RowsDesc(C.Structure):
    """actkv_rows_t: rows of heads with strides."""
    _fields_ = [("base", C.c_void_p), ("stride_layer", C.c_int64), ("stride_row", C.c_int64), ("stride_head", C.c_int64)]


class RopeDesc(C.Structure):
    """actkv_rope_t: which dims turn, by which axis, how fast."""
    _fields_ = [("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("n_axes", C.c_int32), ("section", C.c_int32 * 4),
                ("inv_freq", C.c_void_p)]


class PositionsDesc(C.Structure):
    """actkv_positions_t: a position per (axis, unit, token)."""
    _fields_ = [("base", C.c_void_p), ("stride_axis", C.c_int64), ("stride_unit", C.c_int64)]


class LogitRulesDesc(C.Structure):
    """actkv_logit_rules_t: history, penalties, biases and masks of all requests."""
    _fields_ = [("tokens", C.c_void_p), ("token_stride", C.c_int64), ("hist_len", C.c_void_p), ("prompt_len", C.c_void_p),
                ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p), ("bias_indptr", C.c_void_p),
                ("bias_token", C.c_void_p), ("bias_value", C.c_void_p), ("n_bias", C.c_int32), ("allow", C.c_void_p), ("allow_stride", C.c_int64),
                ("n_allow", C.c_int32), ("allow_row", C.c_void_p)]


class HostStep(C.Structure):
    """actkv_host_step_t: host inputs / outputs, sizes, device staging and scratch of actkv_step_host."""
    _fields_ = ([(n, C.c_void_p) for n in
                 ("q_host", "logits_host", "win_indptr_host", "tok_indptr_host", "logit_indptr_host", "budget_in_host",
                  "page_table_host", "seq_len_host", "free_list_host", "free_count_host",
                  "page_table_out_host", "seq_len_out_host", "free_list_out_host", "free_count_out_host",
                  "budget_out_host", "status_out_host")] +
                [(n, C.c_int32) for n in
                 ("n_q_heads", "sum_win", "max_win", "sum_tok", "max_tok", "n_rows", "vocab", "hist_cap", "max_keep",
                  "causal", "layers_per_call")] +
                [("sm_scale", C.c_float), ("sel_stride", C.c_int64)] +
                [(n, C.c_void_p) for n in
                 ("q_dev", "logits_dev", "win_indptr_dev", "tok_indptr_dev", "logit_indptr_dev", "budget_dev",
                  "keep_indptr_dev", "conf_hist_dev", "hist_len_dev", "lse_dev", "score_dev", "sel_idx_dev")] +
                [("ws_budget", C.c_void_p), ("ws_budget_bytes", C.c_size_t), ("ws_score", C.c_void_p),
                 ("ws_score_bytes", C.c_size_t), ("ws_compact", C.c_void_p), ("ws_compact_bytes", C.c_size_t),
                 ("status_dev", C.c_void_p)])


_lib = None


def load():
    """Open libactkv.so (building it first when nvcc is present and the sources are newer)."""
    global _lib
    if _lib is not None:
        return _lib
    try:
        from . import build as _build
        if os.path.exists(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")):
            _build.build()
    except Exception:
        if not os.path.exists(LIB_PATH):
            raise
    if not os.path.exists(LIB_PATH):
        raise ActKVError("load: libactkv.so is missing; run __graft_entry__.build()", E_CUDA)
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    lib.actkv_version.restype = C.c_char_p
    lib.actkv_budget_workspace_bytes.restype = sz
    lib.actkv_budget_workspace_bytes.argtypes = [i32, i32, i32]
    lib.actkv_budget.restype = i32
    lib.actkv_budget.argtypes = [vp, vp, i32, i32, vp, vp, i32, C.POINTER(BudgetParams), vp, vp, vp, vp, i32,
                                 vp, sz, vp, vp]
    lib.actkv_score_workspace_bytes.restype = sz
    lib.actkv_score_workspace_bytes.argtypes = [C.POINTER(PoolDesc), i32, i32, i32, i32, i32, i32]
    lib.actkv_score.restype = i32
    lib.actkv_score.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, vp, i32, vp, f32, i32,
                                vp, vp, vp, i32, i32, i32, i32, vp, sz, vp, vp]
    lib.actkv_score_lse.restype = i32
    lib.actkv_score_lse.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, vp, i32, f32, i32,
                                    vp, vp, i32, i32, i32, i32, vp, sz, vp, vp]
    lib.actkv_score_accumulate.restype = i32
    lib.actkv_score_accumulate.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, vp, i32, vp, f32,
                                           i32, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp, vp]
    lib.actkv_keep_indptr.restype = i32
    lib.actkv_keep_indptr.argtypes = [vp, vp, i32, vp, vp]
    lib.actkv_select_workspace_bytes.restype = sz
    lib.actkv_select_workspace_bytes.argtypes = [i32, i32, i32]
    lib.actkv_select.restype = i32
    lib.actkv_select.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp, i64, vp, vp, vp, sz, vp, vp]
    lib.actkv_compact_workspace_bytes.restype = sz
    lib.actkv_compact_workspace_bytes.argtypes = [i32, i32]
    lib.actkv_compact.restype = i32
    lib.actkv_compact.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, i64, vp, vp, i32,
                                  vp, sz, vp, vp]
    lib.actkv_keepscore.restype = i32
    lib.actkv_keepscore.argtypes = [vp, vp, i32, i32, i32, f32, f32, vp, vp, vp, vp, vp]
    lib.actkv_compact_inplace.restype = i32
    lib.actkv_compact_inplace.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, i64, vp, vp, i32,
                                          vp, vp, vp]
    lib.actkv_compact_inplace_deferred_workspace_bytes.restype = sz
    lib.actkv_compact_inplace_deferred_workspace_bytes.argtypes = [C.POINTER(PoolDesc), i32, i32, i32]
    for fn in (lib.actkv_compact_inplace_begin, lib.actkv_compact_inplace_end):
        fn.restype = i32
        fn.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, i64, vp, vp, i32, vp, vp, sz, vp, vp]
    lib.actkv_gather_f32.restype = i32
    lib.actkv_gather_f32.argtypes = [vp, i64, vp, vp, i64, vp, i32, i32, i32, vp, i64, vp]
    lib.actkv_step_device.restype = i32
    lib.actkv_step_device.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), C.POINTER(BudgetParams),
                                      C.POINTER(HostStep), i32, vp]
    lib.actkv_step_host.restype = i32
    lib.actkv_step_host.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), C.POINTER(BudgetParams),
                                    C.POINTER(HostStep), vp]
    lib.actkv_compact_noalloc_max_bytes.restype = sz
    lib.actkv_compact_noalloc_max_bytes.argtypes = []
    lib.actkv_compact_noalloc.restype = i32
    lib.actkv_compact_noalloc.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, i64, vp, vp, i32,
                                          vp, vp]
    lib.actkv_compact_begin.restype = i32
    lib.actkv_compact_begin.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, i64, vp, vp, i32, i32, vp,
                                        sz, vp, vp]
    lib.actkv_compact_end.restype = i32
    lib.actkv_compact_end.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, i64, vp, vp, i32, vp, sz,
                                      vp, vp]
    lib.actkv_score_overlap.restype = i32
    lib.actkv_score_overlap.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, vp, i32, vp, f32, i32,
                                        vp, vp, vp, i32, i32, i32, i32, vp, sz, vp, vp, vp]
    lib.actkv_compact_deferred_workspace_bytes.restype = sz
    lib.actkv_compact_deferred_workspace_bytes.argtypes = [C.POINTER(PoolDesc), i32, i32, i32, i32]
    lib.actkv_compact_stats.restype = i32
    lib.actkv_compact_stats.argtypes = [vp, vp, vp]
    lib.actkv_keepscore_select.restype = i32
    lib.actkv_keepscore_select.argtypes = [vp, vp, i32, i32, i32, i32, f32, f32, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp]
    lib.actkv_score_sliding.restype = i32
    lib.actkv_score_sliding.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, vp, i32, vp, f32, i32,
                                        i32, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp, vp]
    lib.actkv_score_path.restype = i32
    lib.actkv_score_path.argtypes = [C.POINTER(PoolDesc), i32, i32, f32, vp, i32]
    lib.actkv_attend_workspace_bytes.restype = sz
    lib.actkv_attend_workspace_bytes.argtypes = [C.POINTER(PoolDesc), i32, i32, i32, i32, i32]
    lib.actkv_attend.restype = i32
    lib.actkv_attend.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, vp, i32, f32, i32, i32, vp, vp,
                                 i32, i32, i32, vp, sz, vp, vp]
    lib.actkv_append.restype = i32
    lib.actkv_append.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, C.POINTER(RowsDesc),
                                 C.POINTER(RowsDesc), C.POINTER(RowsDesc), vp, i32, C.POINTER(RopeDesc), vp, vp, i32, vp, vp]
    lib.actkv_resize.restype = i32
    lib.actkv_resize.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), vp, vp, vp]
    lib.actkv_copy.restype = i32
    lib.actkv_copy.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, vp, vp, vp, i32, i32, vp, vp]
    lib.actkv_logprob.restype = i32
    lib.actkv_logprob.argtypes = [vp, i32, i32, i32, i64, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.actkv_reposition.restype = i32
    lib.actkv_reposition.argtypes = [C.POINTER(PoolDesc), C.POINTER(TablesDesc), i32, i32, C.POINTER(RopeDesc), vp,
                                     C.POINTER(PositionsDesc), C.POINTER(PositionsDesc), vp, i32, i32, vp, vp]
    lib.actkv_penalize.restype = i32
    lib.actkv_penalize.argtypes = [vp, i32, i32, i64, vp, i32, i32, i32, i32, C.POINTER(LogitRulesDesc), vp, i64, vp, vp]
    lib.actkv_sample.restype = i32
    lib.actkv_sample.argtypes = [vp, i32, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.actkv_debug_inject_stall.restype = i32
    lib.actkv_debug_inject_stall.argtypes = [i32, i32]
    _lib = lib
    return lib


# ---------------------------------------------------------------------------------------------
# marshalling helpers


def _ptr(t: Optional[torch.Tensor], dtype=None, name: str = "tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous tensor")
    return t.data_ptr()


def _stream(stream) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _check(fn: str, rc: int):
    if rc != 0:
        raise ActKVError(fn, rc)


def pool_desc(pool: torch.Tensor) -> PoolDesc:
    """Descriptor of a bf16 pool tensor [n_layers, 2, n_pages, page_size, n_kv_heads, head_dim]
    (any strides with a contiguous head dimension)."""
    if pool.dtype != torch.bfloat16 or pool.dim() != 6 or pool.shape[1] != 2 or pool.stride(5) != 1:
        raise TypeError("pool: expected bf16 [NL, 2, n_pages, P, Hkv, D] with contiguous D")
    NL, _, n_pages, P, H, D = pool.shape
    st = pool.stride()
    return PoolDesc(pool.data_ptr(), NL, n_pages, P, H, D, st[0], st[1], st[2], st[3], st[4])


def tables_desc(page_table, seq_len, free_list, free_count) -> TablesDesc:
    R, max_pages = page_table.shape
    return TablesDesc(R, max_pages, _ptr(page_table, torch.int32, "page_table"), _ptr(seq_len, torch.int32, "seq_len"),
                      _ptr(free_list, torch.int32, "free_list"), _ptr(free_count, torch.int32, "free_count"))


# ---------------------------------------------------------------------------------------------
# the entry points


def actkv_version() -> str:
    return load().actkv_version().decode()


def actkv_budget_workspace_bytes(n_rows: int, n_req: int, hist_cap: int) -> int:
    return load().actkv_budget_workspace_bytes(n_rows, n_req, hist_cap)


def actkv_budget(logits, tok_indptr, n_rows, vocab, conf_hist, hist_len, hist_cap, params: BudgetParams,
                 seq_len, budget_in, budget_out, slope_out, n_req, ws, status, stream=None):
    rc = load().actkv_budget(_ptr(logits, torch.float32, "logits"), _ptr(tok_indptr, torch.int32, "tok_indptr"),
                             n_rows, vocab, _ptr(conf_hist, torch.float32, "conf_hist"),
                             _ptr(hist_len, torch.int32, "hist_len"), hist_cap, C.byref(params),
                             _ptr(seq_len, torch.int32, "seq_len"), _ptr(budget_in, torch.int32, "budget_in"),
                             _ptr(budget_out, torch.int32, "budget_out"), _ptr(slope_out, torch.float64, "slope_out"),
                             n_req, _ptr(ws, None, "ws"), ws.numel() * ws.element_size(),
                             _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_budget", rc)


def actkv_score_workspace_bytes(pool: PoolDesc, n_req, n_layers_sub, n_q_heads, sum_win, max_win, max_tok) -> int:
    return load().actkv_score_workspace_bytes(C.byref(pool), n_req, n_layers_sub, n_q_heads, sum_win, max_win, max_tok)


def actkv_score(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, q, win_indptr, n_q_heads, lse_in,
                sm_scale, causal, tok_indptr, score_out, lse_out, sum_win, max_win, sum_tok, max_tok, ws, status,
                stream=None):
    rc = load().actkv_score(C.byref(pool), C.byref(tables), layer_begin, layer_end, _ptr(q, torch.bfloat16, "q"),
                            _ptr(win_indptr, torch.int32, "win_indptr"), n_q_heads,
                            _ptr(lse_in, torch.float32, "lse_in"), float(sm_scale), int(bool(causal)),
                            _ptr(tok_indptr, torch.int32, "tok_indptr"), _ptr(score_out, torch.float32, "score_out"),
                            _ptr(lse_out, torch.float32, "lse_out"), sum_win, max_win, sum_tok, max_tok,
                            _ptr(ws, None, "ws"), ws.numel() * ws.element_size(),
                            _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_score", rc)


def actkv_score_overlap(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, q, win_indptr, n_q_heads, lse_in,
                        sm_scale, causal, tok_indptr, score_out, lse_out, sum_win, max_win, sum_tok, max_tok, ws,
                        pending_compact_ws, status, stream=None):
    rc = load().actkv_score_overlap(C.byref(pool), C.byref(tables), layer_begin, layer_end, _ptr(q, torch.bfloat16, "q"),
                                    _ptr(win_indptr, torch.int32, "win_indptr"), n_q_heads,
                                    _ptr(lse_in, torch.float32, "lse_in"), float(sm_scale), int(bool(causal)),
                                    _ptr(tok_indptr, torch.int32, "tok_indptr"),
                                    _ptr(score_out, torch.float32, "score_out"), _ptr(lse_out, torch.float32, "lse_out"),
                                    sum_win, max_win, sum_tok, max_tok, _ptr(ws, None, "ws"),
                                    ws.numel() * ws.element_size(), _ptr(pending_compact_ws, None, "pending_compact_ws"),
                                    _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_score_overlap", rc)


def actkv_compact_begin(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, sel_idx, sel_stride, keep_indptr,
                        budget, max_keep, ws, status, stream=None, reuse_plan=False):
    rc = load().actkv_compact_begin(C.byref(pool), C.byref(tables), layer_begin, layer_end,
                                    _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride,
                                    _ptr(keep_indptr, torch.int32, "keep_indptr"), _ptr(budget, torch.int32, "budget"),
                                    max_keep, int(bool(reuse_plan)), _ptr(ws, None, "ws"), ws.numel() * ws.element_size(),
                                    _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_compact_begin", rc)


def actkv_compact_end(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, sel_idx, sel_stride, keep_indptr,
                      budget, max_keep, ws, status, stream=None):
    rc = load().actkv_compact_end(C.byref(pool), C.byref(tables), layer_begin, layer_end,
                                  _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride,
                                  _ptr(keep_indptr, torch.int32, "keep_indptr"), _ptr(budget, torch.int32, "budget"),
                                  max_keep, _ptr(ws, None, "ws"), ws.numel() * ws.element_size(),
                                  _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_compact_end", rc)


def actkv_compact_deferred_workspace_bytes(pool: PoolDesc, n_req, max_pages, n_layers_sub, max_keep) -> int:
    return load().actkv_compact_deferred_workspace_bytes(C.byref(pool), n_req, max_pages, n_layers_sub, max_keep)


def actkv_compact_stats(ws, stats, stream=None):
    _check("actkv_compact_stats", load().actkv_compact_stats(_ptr(ws, None, "ws"), _ptr(stats, torch.int32, "stats"),
                                                             _stream(stream)))


def actkv_keepscore_select(score, tok_indptr, sum_tok, max_tok, n_outer, n_req, top_p, lam, n_protect, keep_score,
                           hit_mask, budget, keep_indptr, sel_idx, sel_stride, keep_mask, tie_report, status, stream=None):
    rc = load().actkv_keepscore_select(_ptr(score, torch.float32, "score"), _ptr(tok_indptr, torch.int32, "tok_indptr"),
                                       sum_tok, max_tok, n_outer, n_req, float(top_p), float(lam),
                                       _ptr(n_protect, torch.int32, "n_protect"),
                                       _ptr(keep_score, torch.float32, "keep_score"), _ptr(hit_mask, None, "hit_mask"),
                                       _ptr(budget, torch.int32, "budget"), _ptr(keep_indptr, torch.int32, "keep_indptr"),
                                       _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride, _ptr(keep_mask, None, "keep_mask"),
                                       _ptr(tie_report, None, "tie_report"), _ptr(status, torch.int32, "status"),
                                       _stream(stream))
    _check("actkv_keepscore_select", rc)


def actkv_score_sliding(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, q, win_indptr, n_q_heads, lse_in,
                        sm_scale, causal, window_left, tok_indptr, score_out, lse_out, sum_win, max_win, sum_tok, max_tok,
                        ws, status, stream=None):
    rc = load().actkv_score_sliding(C.byref(pool), C.byref(tables), layer_begin, layer_end, _ptr(q, torch.bfloat16, "q"),
                                    _ptr(win_indptr, torch.int32, "win_indptr"), n_q_heads,
                                    _ptr(lse_in, torch.float32, "lse_in"), float(sm_scale), int(bool(causal)),
                                    int(window_left), _ptr(tok_indptr, torch.int32, "tok_indptr"),
                                    _ptr(score_out, torch.float32, "score_out"), _ptr(lse_out, torch.float32, "lse_out"),
                                    sum_win, max_win, sum_tok, max_tok, _ptr(ws, None, "ws"),
                                    ws.numel() * ws.element_size(), _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_score_sliding", rc)


def actkv_score_path(pool: PoolDesc, n_q_heads, max_win, sm_scale, q, streaming=False) -> int:
    """1: the tensor-core kernels would run, 0: the warp-level (mma.sync) kernels."""
    rc = load().actkv_score_path(C.byref(pool), n_q_heads, max_win, float(sm_scale), _ptr(q, torch.bfloat16, "q"),
                                 int(bool(streaming)))
    if rc < 0:
        raise ActKVError("actkv_score_path", rc)
    return rc


def actkv_debug_inject_stall(after_tile: int, wait_limit_us: int = 0):
    _check("actkv_debug_inject_stall", load().actkv_debug_inject_stall(int(after_tile), int(wait_limit_us)))


def actkv_score_lse(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, q, win_indptr, n_q_heads, sm_scale,
                    causal, tok_indptr, lse_out, sum_win, max_win, sum_tok, max_tok, ws, status, stream=None):
    rc = load().actkv_score_lse(C.byref(pool), C.byref(tables), layer_begin, layer_end, _ptr(q, torch.bfloat16, "q"),
                                _ptr(win_indptr, torch.int32, "win_indptr"), n_q_heads, float(sm_scale),
                                int(bool(causal)), _ptr(tok_indptr, torch.int32, "tok_indptr"),
                                _ptr(lse_out, torch.float32, "lse_out"), sum_win, max_win, sum_tok, max_tok,
                                _ptr(ws, None, "ws"), ws.numel() * ws.element_size(),
                                _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_score_lse", rc)


def actkv_score_accumulate(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, q, win_indptr, n_q_heads, lse_in,
                           sm_scale, causal, tok_indptr, acc_steps, score_io, sum_win, max_win, sum_tok, max_tok, ws,
                           status, stream=None):
    rc = load().actkv_score_accumulate(C.byref(pool), C.byref(tables), layer_begin, layer_end,
                                       _ptr(q, torch.bfloat16, "q"), _ptr(win_indptr, torch.int32, "win_indptr"),
                                       n_q_heads, _ptr(lse_in, torch.float32, "lse_in"), float(sm_scale),
                                       int(bool(causal)), _ptr(tok_indptr, torch.int32, "tok_indptr"),
                                       _ptr(acc_steps, torch.int32, "acc_steps"),
                                       _ptr(score_io, torch.float32, "score_io"), sum_win, max_win, sum_tok, max_tok,
                                       _ptr(ws, None, "ws"), ws.numel() * ws.element_size(),
                                       _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_score_accumulate", rc)


def actkv_keep_indptr(seq_len, budget, n_req, keep_indptr, stream=None):
    rc = load().actkv_keep_indptr(_ptr(seq_len, torch.int32, "seq_len"), _ptr(budget, torch.int32, "budget"), n_req,
                                  _ptr(keep_indptr, torch.int32, "keep_indptr"), _stream(stream))
    _check("actkv_keep_indptr", rc)


def actkv_select_workspace_bytes(n_outer, n_req, max_tok) -> int:
    return load().actkv_select_workspace_bytes(n_outer, n_req, max_tok)


def actkv_select(score, tok_indptr, sum_tok, budget, n_outer, n_req, keep_indptr, sel_idx, sel_stride, keep_mask,
                 tie_report, ws, status, stream=None):
    rc = load().actkv_select(_ptr(score, torch.float32, "score"), _ptr(tok_indptr, torch.int32, "tok_indptr"), sum_tok,
                             _ptr(budget, torch.int32, "budget"), n_outer, n_req,
                             _ptr(keep_indptr, torch.int32, "keep_indptr"), _ptr(sel_idx, torch.int32, "sel_idx"),
                             sel_stride, _ptr(keep_mask, torch.int32, "keep_mask"),
                             _ptr(tie_report, torch.int32, "tie_report"),
                             _ptr(ws, None, "ws"), 0 if ws is None else ws.numel() * ws.element_size(),
                             _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_select", rc)


def actkv_compact_workspace_bytes(n_req, max_pages) -> int:
    return load().actkv_compact_workspace_bytes(n_req, max_pages)


def actkv_compact(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, sel_idx, sel_stride, keep_indptr,
                  budget, max_keep, ws, status, stream=None):
    rc = load().actkv_compact(C.byref(pool), C.byref(tables), layer_begin, layer_end,
                              _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride,
                              _ptr(keep_indptr, torch.int32, "keep_indptr"), _ptr(budget, torch.int32, "budget"),
                              max_keep, _ptr(ws, None, "ws"), ws.numel() * ws.element_size(),
                              _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_compact", rc)


def actkv_compact_inplace(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, sel_idx, sel_stride, keep_indptr,
                          budget, max_keep, new_order, status, stream=None):
    rc = load().actkv_compact_inplace(C.byref(pool), C.byref(tables), layer_begin, layer_end,
                                      _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride,
                                      _ptr(keep_indptr, torch.int32, "keep_indptr"),
                                      _ptr(budget, torch.int32, "budget"), max_keep,
                                      _ptr(new_order, torch.int32, "new_order"),
                                      _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_compact_inplace", rc)


def actkv_compact_inplace_deferred_workspace_bytes(pool: PoolDesc, n_req, n_layers_sub, max_keep) -> int:
    return load().actkv_compact_inplace_deferred_workspace_bytes(C.byref(pool), n_req, n_layers_sub, max_keep)


def _inplace_deferred(fn_name, pool, tables, layer_begin, layer_end, sel_idx, sel_stride, keep_indptr, budget, max_keep,
                      new_order, ws, status, stream):
    rc = getattr(load(), fn_name)(C.byref(pool), C.byref(tables), layer_begin, layer_end,
                                  _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride,
                                  _ptr(keep_indptr, torch.int32, "keep_indptr"), _ptr(budget, torch.int32, "budget"),
                                  max_keep, _ptr(new_order, torch.int32, "new_order"), _ptr(ws, None, "ws"),
                                  ws.numel() * ws.element_size(), _ptr(status, torch.int32, "status"), _stream(stream))
    _check(fn_name, rc)


def actkv_compact_inplace_begin(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, sel_idx, sel_stride,
                                keep_indptr, budget, max_keep, new_order, ws, status, stream=None):
    _inplace_deferred("actkv_compact_inplace_begin", pool, tables, layer_begin, layer_end, sel_idx, sel_stride,
                      keep_indptr, budget, max_keep, new_order, ws, status, stream)


def actkv_compact_inplace_end(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, sel_idx, sel_stride,
                              keep_indptr, budget, max_keep, new_order, ws, status, stream=None):
    _inplace_deferred("actkv_compact_inplace_end", pool, tables, layer_begin, layer_end, sel_idx, sel_stride,
                      keep_indptr, budget, max_keep, new_order, ws, status, stream)


def actkv_keepscore(score, tok_indptr, sum_tok, n_outer, n_req, top_p, lam, n_protect, keep_score, hit_mask, status,
                    stream=None):
    rc = load().actkv_keepscore(_ptr(score, torch.float32, "score"), _ptr(tok_indptr, torch.int32, "tok_indptr"),
                                sum_tok, n_outer, n_req, float(top_p), float(lam),
                                _ptr(n_protect, torch.int32, "n_protect"), _ptr(keep_score, torch.float32, "keep_score"),
                                _ptr(hit_mask, torch.int32, "hit_mask"), _ptr(status, torch.int32, "status"),
                                _stream(stream))
    _check("actkv_keepscore", rc)


def actkv_gather_f32(src, src_stride, tok_indptr, sel_idx, sel_stride, keep_indptr, n_outer, n_req, max_total_keep,
                     dst, dst_stride, stream=None):
    rc = load().actkv_gather_f32(_ptr(src, torch.float32, "src"), src_stride, _ptr(tok_indptr, torch.int32, "tok_indptr"),
                                 _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride,
                                 _ptr(keep_indptr, torch.int32, "keep_indptr"), n_outer, n_req, max_total_keep,
                                 _ptr(dst, torch.float32, "dst"), dst_stride, _stream(stream))
    _check("actkv_gather_f32", rc)


def actkv_step_device(pool: PoolDesc, tables: TablesDesc, params: Optional[BudgetParams], io: HostStep, lse_supplied: bool,
                      stream=None):
    rc = load().actkv_step_device(C.byref(pool), C.byref(tables), None if params is None else C.byref(params),
                                  C.byref(io), int(bool(lse_supplied)), _stream(stream))
    _check("actkv_step_device", rc)


def actkv_step_host(pool: PoolDesc, tables: TablesDesc, params: Optional[BudgetParams], io: HostStep, stream=None):
    """One whole step with host-resident per-step inputs and outputs (synchronises `stream`)."""
    rc = load().actkv_step_host(C.byref(pool), C.byref(tables), None if params is None else C.byref(params),
                                C.byref(io), _stream(stream))
    _check("actkv_step_host", rc)


def actkv_compact_noalloc_max_bytes() -> int:
    return load().actkv_compact_noalloc_max_bytes()


def actkv_compact_noalloc(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, sel_idx, sel_stride,
                          keep_indptr, budget, max_keep, status, stream=None):
    """actkv_compact for callers that cannot allocate the plan scratch: a serving engine that has
    handed all of HBM to its KV pool (cudaMalloc may fail, and it stalls the device), or a host
    without an allocator of its own.  The scratch is a fixed 1 MiB array inside the library, shared
    by every call on the device, so calls that overlap on the GPU race; tables larger than the
    array are refused with ACTKV_E_TOOBIG."""
    rc = load().actkv_compact_noalloc(C.byref(pool), C.byref(tables), layer_begin, layer_end,
                                      _ptr(sel_idx, torch.int32, "sel_idx"), sel_stride,
                                      _ptr(keep_indptr, torch.int32, "keep_indptr"),
                                      _ptr(budget, torch.int32, "budget"), max_keep,
                                      _ptr(status, torch.int32, "status"), _stream(stream))
    _check("actkv_compact_noalloc", rc)


# ---------------------------------------------------------------------------------------------
# decoding between two compression steps
#
# These calls may be made while another device than the tensors' is current; all tensors of a call are on one device.  They
# are made once per layer and token, so the checks take a few tenths of a microsecond per tensor.


def _arg(t, dtype, index, n, name):
    """Address of a contiguous tensor of this type on device `index` with at least n elements (None: null)."""
    if t is None:
        return None
    if t.get_device() != index:
        raise TypeError(f"{name}: on {t.device}, expected cuda:{index}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous tensor")
    if t.numel() < n:
        raise ValueError(f"{name}: {t.numel()} elements, expected at least {n}")
    return t.data_ptr()


def _cuda_index(t, name):
    index = t.get_device()
    if index < 0:
        raise TypeError(f"{name}: expected a CUDA tensor")
    return index


def _call(name, index, stream, *args):
    """Calls the entry point on `stream`, or on the current stream of device `index`, with that device current."""
    raw = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    fn = getattr(_lib or load(), name)
    if torch._C._cuda_getDevice() == index:
        rc = fn(*args, raw)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, raw)
    if rc != 0:
        raise ActKVError(name, rc)


def actkv_attend_workspace_bytes(pool: PoolDesc, n_req, n_layers_sub, n_q_heads, max_win, max_tok) -> int:
    return load().actkv_attend_workspace_bytes(C.byref(pool), n_req, n_layers_sub, n_q_heads, max_win, max_tok)


def actkv_attend(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, q, win_indptr, n_q_heads, sm_scale, causal,
                 window_left, out, lse_out, sum_win, max_win, max_tok, ws, status, stream=None):
    i = _cuda_index(q, "q")
    rows = (layer_end - layer_begin) * sum_win * n_q_heads
    n = rows * pool.head_dim
    _call("actkv_attend", i, stream, pool, tables, layer_begin, layer_end, _arg(q, torch.bfloat16, i, n, "q"),
          _arg(win_indptr, torch.int32, i, tables.n_req + 1, "win_indptr"), n_q_heads, sm_scale, 1 if causal else 0, window_left,
          _arg(out, torch.bfloat16, i, n, "out"), _arg(lse_out, torch.float32, i, rows, "lse_out"), sum_win, max_win, max_tok,
          _arg(ws, torch.uint8, i, 0, "ws"), ws.numel(), _arg(status, torch.int32, i, 4, "status"))


def rows_desc(t: torch.Tensor, name: str = "rows") -> RowsDesc:
    """Descriptor of a bf16 tensor [layers, rows, heads, head_dim] (any strides with a contiguous head dimension)."""
    _cuda_index(t, name)
    st = t.stride()
    if t.dtype is not torch.bfloat16 or len(st) != 4 or (st[3] != 1 and t.shape[3] != 1):
        raise TypeError(f"{name}: expected bf16 [layers, rows, heads, D] with contiguous D")
    return RowsDesc(t.data_ptr(), st[0], st[1], st[2])


def rope_desc(inv_freq: Optional[torch.Tensor], sections, interleaved: bool = False) -> RopeDesc:
    """sections: rotary pairs per axis (1 to 4 axes); inv_freq float32 [sum(sections)] on the device."""
    n = len(sections)
    if not 1 <= n <= 4:
        raise ValueError(f"rope: {n} axes, expected 1 to 4")
    if inv_freq is not None and inv_freq.numel() != sum(sections):
        raise ValueError(f"rope: {inv_freq.numel()} frequencies for {sum(sections)} pairs")
    return RopeDesc(2 * sum(sections), 1 if interleaved else 0, n, (C.c_int32 * 4)(*sections),
                    _ptr(inv_freq, torch.float32, "inv_freq"))


def actkv_append(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, q, k, v, win_indptr, n_q_heads,
                 rope: Optional[RopeDesc], positions, q_out, status, stream=None):
    """q, k, v [layers, rows, heads, head_dim] (strided; q may be None), positions int32 [axes, rows]."""
    i, nls, D = _cuda_index(k, "k"), layer_end - layer_begin, pool.head_dim
    shape = k.shape
    sum_win = shape[1]
    if shape != (nls, sum_win, pool.n_kv_heads, D) or v.shape != shape or (q is not None and q.shape != (nls, sum_win, n_q_heads, D)):
        raise ValueError("actkv_append: q, k and v are [layers, rows, heads, head_dim] of this call and pool")
    if v.get_device() != i or (q is not None and q.get_device() != i):
        raise TypeError(f"q, k, v: expected on cuda:{i}")
    if q is not None and q_out is None:
        raise ValueError("q_out: expected with q")
    n_pos = 0
    if rope is not None and rope.rotary_dim:
        if positions is None:
            raise ValueError("positions: expected with rope")
        n_pos = rope.n_axes * sum_win
    _call("actkv_append", i, stream, pool, tables, layer_begin, layer_end, None if q is None else rows_desc(q, "q"),
          rows_desc(k, "k"), rows_desc(v, "v"), _arg(win_indptr, torch.int32, i, tables.n_req + 1, "win_indptr"), n_q_heads, rope,
          _arg(positions, torch.int32, i, n_pos, "positions"),
          _arg(q_out, torch.bfloat16, i, 0 if q is None else nls * sum_win * n_q_heads * D, "q_out"), sum_win,
          _arg(status, torch.int32, i, 4, "status"))


def actkv_resize(pool: PoolDesc, tables: TablesDesc, new_len, status, stream=None):
    i = _cuda_index(new_len, "new_len")
    _call("actkv_resize", i, stream, pool, tables, _arg(new_len, torch.int32, i, tables.n_req, "new_len"),
          _arg(status, torch.int32, i, 4, "status"))


def actkv_copy(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, src, dst, length, max_len, status, stream=None):
    i, n = _cuda_index(src, "src"), src.numel()
    _call("actkv_copy", i, stream, pool, tables, layer_begin, layer_end, _arg(src, torch.int32, i, n, "src"),
          _arg(dst, torch.int32, i, n, "dst"), _arg(length, torch.int32, i, n, "length"), n, max_len,
          _arg(status, torch.int32, i, 4, "status"))


_LOGIT_TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _result_rows(t, n, width, name):
    """The width of a result buffer [n or more, width] (width None: any); [n] is [n, 1]."""
    shape = None if t is None else t.shape
    if shape == (n,):
        shape = (n, 1)
    if shape is None or len(shape) != 2 or shape[0] < n or (width is not None and shape[1] != width):
        raise ValueError(f"{name}: expected [{n} or more, {'any' if width is None else width}], got {None if shape is None else list(shape)}")
    return shape[1]


def actkv_logprob(logits, given, logprob, entropy, lse, top_logprob, top_index, status, stream=None):
    """logits [rows, vocab] float32 or bf16, rows any distance apart; given int32 [rows, n] or None.  Results: logprob [rows, n],
    entropy and lse [rows], top_logprob and top_index [rows, k], each with room for that many rows or more, or None."""
    i = _cuda_index(logits, "logits")
    kind = _LOGIT_TYPES.get(logits.dtype)
    st = logits.stride()
    if kind is None or len(st) != 2 or (st[1] != 1 and logits.shape[1] != 1):
        raise TypeError("logits: expected float32 or bf16 [rows, vocab] with contiguous rows")
    n, vocab = logits.shape
    n_given = top_k = 0
    if given is not None:
        n_given = _result_rows(given, n, None, "given")
        if given.shape[0] != n:
            raise ValueError(f"given: {given.shape[0]} rows for {n} rows of logits")
        if n_given:
            _result_rows(logprob, n, n_given, "logprob")
    if top_index is not None or top_logprob is not None:
        top_k = _result_rows(top_index, n, None, "top_index")
        _result_rows(top_logprob, n, top_k, "top_logprob")
    _call("actkv_logprob", i, stream, logits.data_ptr(), kind, n, vocab, st[0] if n > 1 else vocab,
          _arg(given, torch.int32, i, 0, "given"), n_given, top_k, _arg(logprob, torch.float32, i, 0, "logprob"),
          _arg(entropy, torch.float32, i, n, "entropy"), _arg(lse, torch.float32, i, n, "lse"),
          _arg(top_logprob, torch.float32, i, 0, "top_logprob"), _arg(top_index, torch.int32, i, 0, "top_index"),
          _arg(status, torch.int32, i, 4, "status"))


def positions_desc(t: torch.Tensor, n_axes: int, n_units: int, name: str = "positions"):
    """Descriptor of int32 positions and the number of tokens that they hold: [tokens] (the same on every axis and for every unit),
    [axes, tokens], or [axes, units, tokens]; one axis or unit stands for all.  The last dim contiguous."""
    if t.dtype is not torch.int32:
        raise TypeError(f"{name}: expected torch.int32, got {t.dtype}")
    shape, st = t.shape, t.stride()
    d = len(shape)
    if not 1 <= d <= 3 or (d > 1 and shape[0] not in (1, n_axes)) or (d == 3 and shape[1] not in (1, n_units)):
        raise ValueError(f"{name}: {list(shape)}, expected [tokens], [{n_axes}, tokens] or [{n_axes}, {n_units}, tokens]")
    if st[-1] != 1 and shape[-1] > 1:
        raise TypeError(f"{name}: expected a contiguous last dimension")
    return PositionsDesc(t.data_ptr(), st[0] if d > 1 and shape[0] > 1 else 0, st[1] if d == 3 and shape[1] > 1 else 0), shape[-1]


def actkv_reposition(pool: PoolDesc, tables: TablesDesc, layer_begin, layer_end, rope: RopeDesc, to_inv_freq, from_pos, to_pos,
                     tok_indptr, max_tok, status, stream=None):
    """from_pos, to_pos: int32 positions (positions_desc), None: a token's index; to_inv_freq float32 [pairs], None: as before.
    tok_indptr [n_req + 1]: where each request's tokens begin in the positions, and how many of them are moved."""
    i = _cuda_index(tok_indptr, "tok_indptr")
    units = (layer_end - layer_begin) * pool.n_kv_heads
    desc, sum_tok = [None, None], 0x7fffffff
    for at, (t, name) in enumerate(((from_pos, "from_pos"), (to_pos, "to_pos"))):
        if t is not None:
            if t.get_device() != i:
                raise TypeError(f"{name}: on {t.device}, expected cuda:{i}")
            desc[at], n = positions_desc(t, rope.n_axes, units, name)
            sum_tok = min(sum_tok, n)
    _call("actkv_reposition", i, stream, pool, tables, layer_begin, layer_end, rope,
          _arg(to_inv_freq, torch.float32, i, rope.rotary_dim // 2, "to_inv_freq"), desc[0], desc[1],
          _arg(tok_indptr, torch.int32, i, tables.n_req + 1, "tok_indptr"), sum_tok, max_tok, _arg(status, torch.int32, i, 4, "status"))


def logit_rules_desc(n_req, tokens=None, hist_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
                     bias_indptr=None, bias_token=None, bias_value=None, allow=None, allow_row=None) -> LogitRulesDesc:
    """tokens int32 [n_req, any]; allow int32 or uint32 [rows, words], 32 tokens a word; the others as actkv_logit_rules_t has them."""
    given = [t for t in (tokens, hist_len, prompt_len, repetition, frequency, presence, bias_indptr, bias_token, bias_value, allow, allow_row)
             if t is not None]
    if not given:
        return LogitRulesDesc()
    i = _cuda_index(given[0], "rules")
    if tokens is not None and (len(tokens.shape) != 2 or tokens.shape[0] != n_req):
        raise ValueError(f"tokens: {list(tokens.shape)}, expected [{n_req}, any]")
    if allow is not None and len(allow.shape) != 2:
        raise ValueError(f"allow: {list(allow.shape)}, expected [rows, words]")
    if tokens is not None and hist_len is None:
        raise ValueError("hist_len: expected with tokens")
    if bias_indptr is not None and (bias_token is None or bias_value is None or bias_token.numel() != bias_value.numel()):
        raise ValueError("bias_token, bias_value: expected with bias_indptr, one value per token")
    if allow is not None and allow.dtype is torch.uint32:
        allow = allow.view(torch.int32)
    desc = LogitRulesDesc(_arg(tokens, torch.int32, i, 0, "tokens"), 0 if tokens is None else tokens.shape[1],
                          _arg(hist_len, torch.int32, i, n_req, "hist_len"), _arg(prompt_len, torch.int32, i, n_req, "prompt_len"),
                          _arg(repetition, torch.float32, i, n_req, "repetition"), _arg(frequency, torch.float32, i, n_req, "frequency"),
                          _arg(presence, torch.float32, i, n_req, "presence"), _arg(bias_indptr, torch.int32, i, n_req + 1, "bias_indptr"),
                          _arg(bias_token, torch.int32, i, 0, "bias_token"), _arg(bias_value, torch.float32, i, 0, "bias_value"), 0 if bias_value is None else bias_value.numel(),
                          _arg(allow, torch.int32, i, 0, "allow"), 0 if allow is None else allow.shape[1], 0 if allow is None else allow.shape[0],
                          _arg(allow_row, torch.int32, i, 0, "allow_row"))
    desc.index, desc.n_req = i, n_req                                       # (what only the tensors know)
    desc.rows = None if allow is None else allow.shape[0] if allow_row is None else allow_row.numel()
    return desc


def _logit_rows(t, index, name):
    """Type code, rows, vocabulary and row stride of logits on this device."""
    kind, st = _LOGIT_TYPES.get(t.dtype), t.stride()
    if kind is None or len(st) != 2 or (st[1] != 1 and t.shape[1] != 1):
        raise TypeError(f"{name}: expected float32 or bf16 [rows, vocab] with contiguous rows")
    if t.get_device() != index:
        raise TypeError(f"{name}: on {t.device}, expected cuda:{index}")
    n, vocab = t.shape
    return kind, n, vocab, st[0] if n > 1 else vocab


def actkv_penalize(logits, win_indptr, n_req, rules: LogitRulesDesc, max_win, max_hist, out, status, stream=None):
    """logits [rows, vocab] float32 or bf16, rows any distance apart; out: the same tensor (in place), or one of its shape and type."""
    i = _cuda_index(logits, "logits")
    kind, n, vocab, stride = _logit_rows(logits, i, "logits")
    if getattr(rules, "index", i) != i:
        raise TypeError(f"rules: on cuda:{rules.index}, expected cuda:{i}")
    if getattr(rules, "n_req", 0) not in (0, n_req):
        raise ValueError(f"rules: of {rules.n_req} requests, win_indptr: of {n_req}")
    if getattr(rules, "rows", None) is not None and rules.rows < n:
        raise ValueError(f"allow: masks for {rules.rows} rows, logits: {n}")
    to, out_stride = logits.data_ptr(), stride
    if out is not logits:
        if out.dtype is not logits.dtype or out.shape != logits.shape:
            raise ValueError(f"out: expected {logits.dtype} {list(logits.shape)}, got {out.dtype} {list(out.shape)}")
        to, out_stride = out.data_ptr(), _logit_rows(out, i, "out")[3]
    _call("actkv_penalize", i, stream, logits.data_ptr(), kind, vocab, stride, _arg(win_indptr, torch.int32, i, n_req + 1, "win_indptr"), n_req,
          n, max_win, max_hist, rules, to, out_stride, _arg(status, torch.int32, i, 4, "status"))


def actkv_sample(logits, u, temperature, top_k, top_p, min_p, token, logprob, kept, status, stream=None):
    """logits [rows, vocab] float32 or bf16, rows any distance apart; u, temperature, top_p, min_p float32 and top_k int32 [rows] (None: 1, 1, 0,
    0); results token int32, logprob float32, kept int32 with room for that many rows (the last two may be None)."""
    i = _cuda_index(logits, "logits")
    kind, n, vocab, stride = _logit_rows(logits, i, "logits")
    f32, i32 = torch.float32, torch.int32
    _call("actkv_sample", i, stream, logits.data_ptr(), kind, n, vocab, stride, _arg(u, f32, i, n, "u"),
          _arg(temperature, f32, i, n, "temperature"), _arg(top_k, i32, i, n, "top_k"), _arg(top_p, f32, i, n, "top_p"),
          _arg(min_p, f32, i, n, "min_p"), _arg(token, i32, i, n, "token"), _arg(logprob, f32, i, n, "logprob"), _arg(kept, i32, i, n, "kept"),
          _arg(status, i32, i, 4, "status"))
