"""Binding of libslkv.so: the same entry points as include/slkv.h, argument marshalling only.

Tensors are torch tensors (device memory and streams come from torch); every step of the method runs in
the library's kernels.  There is no fallback: if the shared library is missing, lib() raises.
Calls that a program makes per layer go through a small C module (csrc/slkv_pycall.c) that converts tensors, lists and
structures itself: about 1 us a call, against 8 us through ctypes.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import List, Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libslkv.so")

SLKV_OK = 0
ERR = {"NULL_PTR": -1, "BAD_SHAPE": -2, "BAD_DTYPE": -3, "BAD_ALIGN": -4, "BUDGET_SUM": -5, "NEG_INF_SC": -6,
       "CAPACITY": -7, "WORKSPACE": -8, "CUDA": -9, "DEVICE_TIMEOUT": -10}
SLKV_F32, SLKV_BF16 = 0, 1
SLKV_POOL_MAX, SLKV_POOL_AVG = 0, 1
SLKV_HISTORY, SLKV_ALL_CAUSAL = 0, 1
SLKV_LSE_LN, SLKV_LSE_LOG2 = 0, 1
SLKV_PATH_AUTO, SLKV_PATH_SIMT, SLKV_PATH_TENSOR = 0, 1, 2
_DTYPES = {torch.float32: SLKV_F32, torch.bfloat16: SLKV_BF16}


class SlkvParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "n_q_heads", "n_kv_heads", "head_dim", "window", "pool_kernel",
                                         "dtype", "pool_mode", "softmax_domain", "score_path", "lse_units",
                                         "history_only")] + \
               [(n, C.c_int64) for n in ("k_stride_tok", "k_stride_head", "v_stride_tok", "v_stride_head",
                                         "q_stride_seq", "q_stride_row", "q_stride_head")]


class SlkvAllocOptions(C.Structure):
    _fields_ = [("head_normaliser", C.c_int32), ("rounding", C.c_int32), ("cap", C.c_int64)]


class SlkvQ4Cache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "n_kv_heads", "head_dim", "reserved")] + [("capacity_rows", C.c_int64)] + \
               [(n, C.c_void_p) for n in ("records", "pos", "weight", "starts", "lens")]


class SlkvQ4AttendParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_tokens", "dtype", "lse_units")] + \
               [(n, C.c_float) for n in ("scale", "softcap", "weight_decay")] + [("reserved", C.c_int32)] + \
               [(n, C.c_int64) for n in ("q_stride_seq", "q_stride_tok", "q_stride_head", "o_stride_seq", "o_stride_tok",
                                         "o_stride_head")]


class SlkvPromptParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "n_q_heads", "n_kv_heads", "head_dim", "window", "dtype", "lse_units")] + \
               [("scale", C.c_float)] + \
               [(n, C.c_int64) for n in ("q_stride_tok", "q_stride_head", "k_stride_tok", "k_stride_head", "v_stride_tok",
                                         "v_stride_head", "o_stride_tok", "o_stride_head")]


class SlkvPagedCache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_seqs", "n_kv_heads", "head_dim", "dtype", "page_rows", "n_pages",
                                         "max_pages")] + \
               [(n, C.c_void_p) for n in ("k_pages", "v_pages", "tables", "lens", "free_pages", "n_free")]


class SlkvPagedAttendParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_tokens", "layer", "has_new", "lse_units")] + [("scale", C.c_float)] + \
               [(f"{x}_stride_{y}", C.c_int64) for x in "qokv" for y in ("seq", "tok", "head")]


SLKV_NORM_GLOBAL, SLKV_NORM_WITHIN_LAYER = 0, 1
SLKV_PAGED_LENGTHS, SLKV_PAGED_OFFSETS, SLKV_PAGED_ADD = 0, 1, 2
SLKV_ROUND_SUM_EXACT, SLKV_ROUND_PAPER = 0, 1


class SlkvError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().slkv_strerror(code).decode()
        if code == ERR["CUDA"]:
            msg += f" (cudaError {lib().slkv_last_cuda_error()})"
        super().__init__(f"{where}: {msg}")


_lib = None


def lib() -> C.CDLL:
    """The loaded shared library (loads it on first use; raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2508_15806_b200.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        vp, i32p, i64, i32, sz = C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
        pp = C.POINTER(SlkvParams)
        L.slkv_strerror.restype = C.c_char_p
        L.slkv_strerror.argtypes = [C.c_int]
        L.slkv_last_cuda_error.restype = C.c_int
        L.slkv_last_launch_count.restype = C.c_int
        L.slkv_version.restype = C.c_int
        L.slkv_alloc_budgets.restype = C.c_int
        L.slkv_alloc_budgets.argtypes = [vp, i32, i32, i32, i64, vp, vp, vp]
        L.slkv_alloc_budgets_ex.restype = C.c_int
        L.slkv_alloc_budgets_ex.argtypes = [vp, i32, i32, i32, i64, C.POINTER(SlkvAllocOptions), vp, vp, vp]
        L.slkv_behavior_scores.restype = C.c_int
        L.slkv_behavior_scores.argtypes = [vp, i64, i32, i64, vp, i32, i64, vp, i32, i64, vp, vp, vp, vp]
        L.slkv_workspace_bytes.restype = sz
        L.slkv_workspace_bytes.argtypes = [pp, i32p]
        L.slkv_pooled_elems.restype = i64
        L.slkv_pooled_elems.argtypes = [pp, i32p]
        L.slkv_packed_rows_upper_bound.restype = i64
        L.slkv_packed_rows_upper_bound.argtypes = [pp, i32p]
        L.slkv_score.restype = C.c_int
        L.slkv_score.argtypes = [pp, vp, vp, vp, i32p, vp, vp, vp, vp, sz, vp]
        L.slkv_row_lse.restype = C.c_int
        L.slkv_row_lse.argtypes = [pp, vp, vp, vp, i32p, vp, vp, vp, sz, vp]
        L.slkv_debug_expire_next_wait.restype = C.c_int
        L.slkv_debug_expire_next_wait.argtypes = [C.c_int]
        L.slkv_debug_list_way.restype = C.c_int
        L.slkv_debug_list_way.argtypes = [C.c_int]
        L.slkv_compress.restype = C.c_int
        L.slkv_compress.argtypes = [pp, vp, vp, vp, vp, i32p, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, sz, vp]
        L.slkv_compress_overlapped.restype = C.c_int
        L.slkv_compress_overlapped.argtypes = L.slkv_compress.argtypes
        L.slkv_workspace_bytes_overlapped.restype = sz
        L.slkv_workspace_bytes_overlapped.argtypes = [pp, i32p]
        L.slkv_join.restype = C.c_int
        L.slkv_join.argtypes = [vp]
        L.slkv_compress_host_arena_bytes.restype = sz
        L.slkv_compress_host_arena_bytes.argtypes = [pp, i32p, i64]
        L.slkv_compress_host.restype = C.c_int
        L.slkv_compress_host.argtypes = [pp, vp, vp, vp, i32p, vp, vp, vp, i64, vp, vp, C.POINTER(C.c_int64),
                                         vp, sz, vp]
        L.slkv_score_noalloc.restype = C.c_int
        L.slkv_score_noalloc.argtypes = [pp, vp, vp, vp, i32p, vp, vp, vp, vp]
        L.slkv_noalloc_scratch_bytes.restype = sz
        L.slkv_noalloc_last_cuda_error.restype = C.c_int
        L.slkv_profile_enable.restype = C.c_int
        L.slkv_profile_enable.argtypes = [C.c_int]
        L.slkv_profile_collect.restype = C.c_int
        L.slkv_profile_collect.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_int32), C.c_int32]
        L.slkv_kernel_name.restype = C.c_char_p
        L.slkv_kernel_name.argtypes = [C.c_int]
        L.slkv_kernel_count.restype = C.c_int
        L.slkv_trace_set_buffer.restype = C.c_int
        L.slkv_trace_set_buffer.argtypes = [C.c_void_p, C.c_size_t]
        i32 = C.c_int32
        L.slkv_cp_merge_lse.restype = C.c_int
        L.slkv_cp_merge_lse.argtypes = [pp, vp, i32, vp, vp]
        L.slkv_cp_select_init.restype = C.c_int
        L.slkv_cp_select_init.argtypes = [vp, i32, i32, i64, vp, vp, vp]
        L.slkv_cp_histogram.restype = C.c_int
        L.slkv_cp_histogram.argtypes = [vp, i32, i64, i32, i32, i32, vp, vp, vp]
        L.slkv_cp_descend.restype = C.c_int
        L.slkv_cp_descend.argtypes = [vp, i32, i32, vp, vp, vp]
        L.slkv_cp_local_ties.restype = C.c_int
        L.slkv_cp_local_ties.argtypes = [vp, vp, i32, vp, vp]
        L.slkv_cp_workspace_bytes.restype = sz
        L.slkv_cp_workspace_bytes.argtypes = [i32, i32, i64]
        L.slkv_cp_emit.restype = C.c_int
        L.slkv_cp_emit.argtypes = [pp, vp, vp, i64, vp, i64, i32, i32, i64, vp, vp, vp, i32, i32, i32, i64, vp, vp, i64,
                                   vp, vp, vp, vp, sz, vp]
        cp, ap = C.POINTER(SlkvQ4Cache), C.POINTER(SlkvQ4AttendParams)
        L.slkv_q4_record_bytes.restype = sz
        L.slkv_q4_record_bytes.argtypes = [i32]
        L.slkv_q4_pack.restype = C.c_int
        L.slkv_q4_pack.argtypes = [cp, i32, vp, vp, i64, vp, vp, vp, vp]
        L.slkv_q4_append.restype = C.c_int
        L.slkv_q4_append.argtypes = [cp, i32, vp, vp, i32, i64, i64, i64, i64, i64, i64, vp, vp, vp, vp]
        L.slkv_q4_unpack.restype = C.c_int
        L.slkv_q4_unpack.argtypes = [cp, i32, vp, i64, vp, vp, vp]
        L.slkv_q4_attend_workspace_bytes.restype = sz
        L.slkv_q4_attend_workspace_bytes.argtypes = [cp, ap, i32]
        L.slkv_q4_attend.restype = C.c_int
        L.slkv_q4_attend.argtypes = [cp, ap, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
        L.slkv_q4_evict_workspace_bytes.restype = sz
        L.slkv_q4_evict_workspace_bytes.argtypes = [cp]
        L.slkv_q4_evict.restype = C.c_int
        L.slkv_q4_evict.argtypes = [cp, cp, vp, i32, vp, vp, vp, sz, vp]
        rp, gp, tp = C.POINTER(SlkvPromptParams), C.POINTER(SlkvPagedCache), C.POINTER(SlkvPagedAttendParams)
        L.slkv_prompt_attend_workspace_bytes.restype = sz
        L.slkv_prompt_attend_workspace_bytes.argtypes = [rp, i32p, i32p]
        L.slkv_prompt_attend.restype = C.c_int
        L.slkv_prompt_attend.argtypes = [rp, vp, vp, vp, vp, i32p, vp, i32p, vp, vp, vp, vp, sz, vp]
        L.slkv_paged_plan.restype = C.c_int
        L.slkv_paged_plan.argtypes = [gp, i32, vp, vp, i64, i32, vp, vp, vp, vp, vp]
        L.slkv_paged_write.restype = C.c_int
        L.slkv_paged_write.argtypes = [gp, vp, vp, i32, i32, i32, i64, i64, i64, i64, i64, i64, vp, i32, vp, vp]
        L.slkv_paged_attend_workspace_bytes.restype = sz
        L.slkv_paged_attend_workspace_bytes.argtypes = [gp, tp]
        L.slkv_paged_attend.restype = C.c_int
        L.slkv_paged_attend.argtypes = [gp, tp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


class _EntryPoints(dict):
    """Entry point name -> callable(stream, *args); filled on first use."""

    def __missing__(self, name: str):
        address = C.cast(getattr(lib(), name), C.c_void_p).value
        from ._slkv_call import call
        self[name] = fn = functools.partial(call, address)
        return fn


_fn = _EntryPoints()


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _cu_host(cu_seqlens: Sequence[int]):
    arr = (C.c_int32 * len(cu_seqlens))(*[int(x) for x in cu_seqlens])
    return arr


def _cu_list(cu_seqlens: Sequence[int]):
    return cu_seqlens if type(cu_seqlens) in (list, tuple) else [int(x) for x in cu_seqlens]


def make_params(q_win: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor], window: int, pool_kernel: int,
                pool_mode: int = SLKV_POOL_MAX, score_path: int = SLKV_PATH_AUTO,
                softmax_domain: int = SLKV_HISTORY, lse_units: int = SLKV_LSE_LN) -> SlkvParams:
    """Shapes and strides from the tensors: q_win [n_seqs, w, Hq, d], k / v [T, Hkv, d] (last dim contiguous)."""
    assert q_win.dim() == 4 and k.dim() == 3 and q_win.stride(3) == 1 and k.stride(2) == 1
    if v is None:
        v = k
    dt = _DTYPES[k.dtype]
    assert q_win.dtype == k.dtype == v.dtype
    (n_seqs, _, n_q_heads, _), (_, n_kv_heads, head_dim) = q_win.shape, k.shape
    (k_tok, k_head, _), (v_tok, v_head, _), (q_seq, q_row, q_head, _) = k.stride(), v.stride(), q_win.stride()
    return SlkvParams(n_seqs, n_q_heads, n_kv_heads, head_dim, window, pool_kernel, dt, pool_mode, softmax_domain, score_path,
                      lse_units, 0, k_tok, k_head, v_tok, v_head, q_seq, q_row, q_head)


def slkv_version() -> int:
    return lib().slkv_version()


def slkv_last_launch_count() -> int:
    return lib().slkv_last_launch_count()


def slkv_alloc_budgets(inf_sc: torch.Tensor, fixed: int, total: int, budgets: Optional[torch.Tensor] = None,
                       status: Optional[torch.Tensor] = None, stream=None,
                       options: Optional[SlkvAllocOptions] = None) -> torch.Tensor:
    """inf_sc: CUDA float32 [n_layers, n_heads] -> CUDA int32 budgets of the same shape (slkv_alloc_budgets, or
    slkv_alloc_budgets_ex when `options` is given)."""
    assert inf_sc.is_cuda and inf_sc.dtype == torch.float32 and inf_sc.dim() == 2 and inf_sc.is_contiguous()
    if budgets is None:
        budgets = torch.empty(inf_sc.shape, dtype=torch.int32, device=inf_sc.device)
    n_layers, n_heads = inf_sc.shape
    if options is not None:
        rc = _fn["slkv_alloc_budgets_ex"](stream, inf_sc, n_layers, n_heads, int(fixed), int(total), options, budgets,
                                          status)
        if rc != SLKV_OK:
            raise SlkvError(rc, "slkv_alloc_budgets_ex")
        return budgets
    rc = _fn["slkv_alloc_budgets"](stream, inf_sc, n_layers, n_heads, int(fixed), int(total), budgets, status)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_alloc_budgets")
    return budgets


def slkv_behavior_scores(attn: torch.Tensor, needle_idx: torch.Tensor, topk_idx: torch.Tensor, stream=None):
    """Algorithm 1 for a batch: attn CUDA float32 [n_rows, row_len]; needle_idx / topk_idx CUDA int32 [n_rows, n] or
    [n] (one list for all rows), entries < 0 are padding.  Returns (SF_sc, LG_sc, INF_sc), CUDA float32 [n_rows]."""
    n_rows, row_len = attn.shape
    row_stride, one = attn.stride()
    assert attn.is_cuda and attn.dtype == torch.float32 and one == 1
    for t in (needle_idx, topk_idx):
        assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.dim() in (1, 2)
    sf = torch.empty(n_rows, dtype=torch.float32, device=attn.device)      # three tensors: cheaper than views of one
    lg, inf = torch.empty_like(sf), torch.empty_like(sf)
    nn, tn = needle_idx.size(-1), topk_idx.size(-1)
    rc = _fn["slkv_behavior_scores"](stream, attn, n_rows, row_len, row_stride, needle_idx, nn,
                                     nn if needle_idx.dim() == 2 else 0, topk_idx, tn, tn if topk_idx.dim() == 2 else 0,
                                     sf, lg, inf)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_behavior_scores")
    return sf, lg, inf


def slkv_workspace_bytes(params: SlkvParams, cu_seqlens: Sequence[int]) -> int:
    return int(lib().slkv_workspace_bytes(C.byref(params), _cu_host(cu_seqlens)))


def slkv_pooled_elems(params: SlkvParams, cu_seqlens: Sequence[int]) -> int:
    return int(lib().slkv_pooled_elems(C.byref(params), _cu_host(cu_seqlens)))


def slkv_packed_rows_upper_bound(params: SlkvParams, cu_seqlens: Sequence[int]) -> int:
    return int(lib().slkv_packed_rows_upper_bound(C.byref(params), _cu_host(cu_seqlens)))


def new_workspace(params: SlkvParams, cu_seqlens: Sequence[int], device) -> torch.Tensor:
    n = slkv_workspace_bytes(params, cu_seqlens)
    if n == 0:
        raise SlkvError(ERR["BAD_SHAPE"], "slkv_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _lse(lse: Optional[torch.Tensor], params: SlkvParams) -> Optional[torch.Tensor]:
    if lse is None:
        return None
    assert lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous()
    assert lse.numel() == params.n_seqs * params.n_q_heads * params.window, "lse is [n_seqs, n_q_heads, window]"
    return lse


def slkv_score(params: SlkvParams, q_win: torch.Tensor, k: torch.Tensor, cu_dev: torch.Tensor,
               cu_seqlens: Sequence[int], pooled: torch.Tensor, workspace: torch.Tensor,
               status: Optional[torch.Tensor] = None, stream=None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
    rc = _fn["slkv_score"](stream, params, q_win, k, cu_dev, _cu_list(cu_seqlens), _lse(lse, params), pooled, status,
                           workspace, workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_score")
    return pooled


def slkv_row_lse(params: SlkvParams, q_win: torch.Tensor, k: torch.Tensor, cu_dev: torch.Tensor,
                 cu_seqlens: Sequence[int], lse_out: torch.Tensor, workspace: torch.Tensor,
                 status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """lse_out: CUDA float32 [n_seqs, n_q_heads, window], the window rows' log-sum-exp in params.lse_units."""
    _lse(lse_out, params)
    rc = _fn["slkv_row_lse"](stream, params, q_win, k, cu_dev, _cu_list(cu_seqlens), lse_out, status, workspace,
                             workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_row_lse")
    return lse_out


def slkv_debug_expire_next_wait(on=True) -> None:
    """False / 0: off; True / 1: the wait for the statistics; 2: the wait for their clearing; of a layer in one launch, 3: the wait
    for the row sums, 4: the wait for the votes; 5: attention over the 4-bit cache, a wait for rows, or attention of prompts and over
    pages, a wait for probabilities."""
    lib().slkv_debug_expire_next_wait(int(on))


def slkv_debug_list_way(way=0) -> None:
    """Lists this thread sends out without pooled scores: 1 one product with every key, 2 two, 0 by the library's rule."""
    lib().slkv_debug_list_way(int(way))


def slkv_score_noalloc(params: SlkvParams, q_win: torch.Tensor, k: torch.Tensor, cu_dev: torch.Tensor,
                       cu_seqlens: Sequence[int], pooled: torch.Tensor, status: Optional[torch.Tensor] = None,
                       stream=None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
    """slkv_score for callers that cannot allocate: the scratch is a fixed array inside the library
    (slkv_noalloc_scratch_bytes() bytes); larger shapes raise SLKV_ERR_WORKSPACE."""
    rc = _fn["slkv_score_noalloc"](stream, params, q_win, k, cu_dev, _cu_list(cu_seqlens), _lse(lse, params), pooled,
                                   status)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_score_noalloc")
    return pooled


def slkv_noalloc_scratch_bytes() -> int:
    return int(lib().slkv_noalloc_scratch_bytes())


def slkv_compress(params: SlkvParams, q_win, k, v, cu_dev, cu_seqlens: Sequence[int], budgets, k_out, v_out,
                  offsets, kept_idx, workspace, pooled: Optional[torch.Tensor] = None,
                  status: Optional[torch.Tensor] = None, stream=None, lse: Optional[torch.Tensor] = None) -> None:
    rc = _fn["slkv_compress"](stream, params, q_win, k, v, cu_dev, _cu_list(cu_seqlens), budgets, _lse(lse, params),
                              k_out, v_out, k_out.size(0), offsets, kept_idx, pooled, status, workspace,
                              workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_compress")


def slkv_compress_overlapped(params: SlkvParams, q_win, k, v, cu_dev, cu_seqlens: Sequence[int], budgets, k_out,
                             v_out, offsets, kept_idx, workspace, pooled: Optional[torch.Tensor] = None,
                             status: Optional[torch.Tensor] = None, stream=None,
                             lse: Optional[torch.Tensor] = None) -> None:
    """slkv_compress with successive calls overlapped on the GPU; outputs are valid behind slkv_join()."""
    rc = _fn["slkv_compress_overlapped"](stream, params, q_win, k, v, cu_dev, _cu_list(cu_seqlens), budgets,
                                         _lse(lse, params), k_out, v_out, k_out.size(0), offsets, kept_idx, pooled,
                                         status, workspace, workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_compress_overlapped")


def slkv_workspace_bytes_overlapped(params: SlkvParams, cu_seqlens: Sequence[int]) -> int:
    return int(lib().slkv_workspace_bytes_overlapped(C.byref(params), _cu_host(cu_seqlens)))


def slkv_join(stream=None) -> None:
    rc = _fn["slkv_join"](stream)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_join")


def slkv_compress_host_arena_bytes(params: SlkvParams, cu_seqlens: Sequence[int], capacity_rows: int) -> int:
    return int(lib().slkv_compress_host_arena_bytes(C.byref(params), _cu_host(cu_seqlens), int(capacity_rows)))


def slkv_compress_host(params: SlkvParams, q_win, k, v, cu_seqlens: Sequence[int], budgets, k_out, v_out, offsets,
                       kept_idx, arena: torch.Tensor, stream=None) -> int:
    """All tensors except `arena` are HOST tensors (pinned for speed); returns the number of packed rows."""
    for t in (q_win, k, v, budgets, k_out, v_out, offsets, kept_idx):
        assert not t.is_cuda and t.is_contiguous()
    assert arena.is_cuda
    rows = C.c_int64(0)
    rc = _fn["slkv_compress_host"](stream, params, q_win, k, v, _cu_list(cu_seqlens), budgets, k_out, v_out,
                                   k_out.size(0), offsets, kept_idx, rows, arena, arena.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_compress_host")
    return int(rows.value)


def slkv_profile_enable(on) -> None:
    """False / 0: off; True / 1: every kernel (one stream); 2: the score kernels only."""
    lib().slkv_profile_enable(int(on))


def slkv_profile_collect() -> dict:
    """{kernel name: (total milliseconds, launches)} since the last collect, for kernels that ran."""
    n = lib().slkv_kernel_count()
    ms = (C.c_float * n)()
    cnt = (C.c_int32 * n)()
    rc = lib().slkv_profile_collect(ms, cnt, n)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_profile_collect")
    return {lib().slkv_kernel_name(i).decode(): (float(ms[i]), int(cnt[i])) for i in range(n) if cnt[i] > 0}


def slkv_trace_set_buffer(buf: Optional[torch.Tensor]) -> None:
    """buf: CUDA int64 tensor that receives the score kernels' timeline stamps, or None to switch tracing off."""
    if buf is None:
        lib().slkv_trace_set_buffer(None, 0)
    else:
        lib().slkv_trace_set_buffer(buf.data_ptr(), buf.numel() * buf.element_size())


# ---- context-parallel selection (one sequence's keys split over ranks): thin wrappers, see include/slkv.h ------------
def _check(rc: int, what: str) -> None:
    if rc != SLKV_OK:
        raise SlkvError(rc, what)


def slkv_cp_merge_lse(params: SlkvParams, lse_parts: torch.Tensor, lse_out: torch.Tensor, stream=None) -> torch.Tensor:
    """lse_parts: CUDA float32 [n_parts, n_q_heads, window] (contiguous); lse_out: [1, n_q_heads, window]."""
    _check(_fn["slkv_cp_merge_lse"](stream, params, lse_parts, lse_parts.size(0), lse_out), "slkv_cp_merge_lse")
    return lse_out


def slkv_cp_row_lse(params: SlkvParams, q_win: torch.Tensor, k: torch.Tensor, cu_dev: torch.Tensor, cu_seqlens: Sequence[int],
                    lse_out: torch.Tensor, zeroed_workspace, workspace_bytes: int, status: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """slkv_row_lse on a workspace (a tensor or an address) that is zero throughout."""
    _lse(lse_out, params)
    _check(_fn["slkv_cp_row_lse"](stream, params, q_win, k, cu_dev, _cu_list(cu_seqlens), lse_out, status, zeroed_workspace,
                                  workspace_bytes), "slkv_cp_row_lse")
    return lse_out


def slkv_score_at(params: SlkvParams, q_win: torch.Tensor, k: torch.Tensor, cu_dev: torch.Tensor, cu_seqlens: Sequence[int],
                  pooled: torch.Tensor, workspace: int, workspace_bytes: int, status: Optional[torch.Tensor] = None, stream=None,
                  lse: Optional[torch.Tensor] = None) -> torch.Tensor:
    """slkv_score with the workspace given as an address."""
    _check(_fn["slkv_score"](stream, params, q_win, k, cu_dev, _cu_list(cu_seqlens), _lse(lse, params), pooled, status, workspace,
                             workspace_bytes), "slkv_score")
    return pooled


def slkv_cp_select_init(budgets: torch.Tensor, window: int, seq_len: int, prefix: torch.Tensor, need: torch.Tensor,
                        stream=None) -> None:
    _check(_fn["slkv_cp_select_init"](stream, budgets, budgets.numel(), int(window), int(seq_len), prefix, need),
           "slkv_cp_select_init")


def slkv_cp_histogram(pooled: torch.Tensor, n_kv_heads: int, row_stride: int, own_begin: int, own_count: int, level: int,
                      prefix: torch.Tensor, hist: torch.Tensor, stream=None) -> torch.Tensor:
    _check(_fn["slkv_cp_histogram"](stream, pooled, int(n_kv_heads), int(row_stride), int(own_begin), int(own_count),
                                    int(level), prefix, hist), "slkv_cp_histogram")
    return hist


def slkv_cp_descend(hist: torch.Tensor, level: int, prefix: torch.Tensor, need: torch.Tensor, stream=None) -> None:
    _check(_fn["slkv_cp_descend"](stream, hist, prefix.numel(), int(level), prefix, need), "slkv_cp_descend")


def slkv_cp_local_ties(hist_local: torch.Tensor, prefix: torch.Tensor, ties: torch.Tensor, stream=None) -> torch.Tensor:
    _check(_fn["slkv_cp_local_ties"](stream, hist_local, prefix, prefix.numel(), ties), "slkv_cp_local_ties")
    return ties


def slkv_cp_step(budgets: Optional[torch.Tensor], n_kv_heads: int, window: int, seq_len: int, level: int, state,
                 hist_sum: Optional[torch.Tensor], pooled: torch.Tensor, row_stride: int, own_begin: int, own_count: int,
                 hist: Optional[torch.Tensor], totals: Optional[torch.Tensor] = None, clear=None, clear_bytes: int = 0,
                 workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    """One launch between two collectives (see include/slkv.h).  state, clear and workspace: tensors or addresses."""
    _check(_fn["slkv_cp_step"](stream, budgets, n_kv_heads, window, seq_len, level, state, hist_sum, pooled, row_stride,
                               own_begin, own_count, hist, totals, clear, clear_bytes, workspace, workspace_bytes),
           "slkv_cp_step")


def slkv_cp_emit_counted(params: SlkvParams, k: torch.Tensor, v: torch.Tensor, rows: int, pooled: torch.Tensor,
                         row_stride: int, own_begin: int, own_count: int, pos0: int, threshold, need,
                         ties_all: torch.Tensor, part: int, window_rows: int, window_pos0: int, totals: torch.Tensor,
                         k_out: torch.Tensor, v_out: torch.Tensor, offsets: torch.Tensor, kept_idx: torch.Tensor,
                         workspace, workspace_bytes: int, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """slkv_cp_emit behind slkv_cp_step's level 3.  threshold, need and workspace: tensors or addresses."""
    _check(_fn["slkv_cp_emit_counted"](stream, params, k, v, rows, pooled, row_stride, own_begin, own_count, pos0,
                                       threshold, need, ties_all, ties_all.size(0), part, window_rows, window_pos0,
                                       totals, k_out, v_out, k_out.size(0), offsets, kept_idx, status, workspace,
                                       workspace_bytes), "slkv_cp_emit_counted")


def slkv_cp_workspace_bytes(n_kv_heads: int, own_count: int, capacity_rows: int) -> int:
    return int(lib().slkv_cp_workspace_bytes(int(n_kv_heads), int(own_count), int(capacity_rows)))


def slkv_cp_emit(params: SlkvParams, k: torch.Tensor, v: torch.Tensor, rows: int, pooled: torch.Tensor, row_stride: int,
                 own_begin: int, own_count: int, pos0: int, threshold: torch.Tensor, need: torch.Tensor,
                 ties_all: torch.Tensor, part: int, window_rows: int, window_pos0: int, k_out: torch.Tensor,
                 v_out: torch.Tensor, offsets: torch.Tensor, kept_idx: torch.Tensor, workspace: torch.Tensor,
                 status: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(_fn["slkv_cp_emit"](stream, params, k, v, int(rows), pooled, int(row_stride), int(own_begin), int(own_count),
                               int(pos0), threshold, need, ties_all, ties_all.size(0), int(part), int(window_rows),
                               int(window_pos0), k_out, v_out, k_out.size(0), offsets, kept_idx, status, workspace,
                               workspace.numel()), "slkv_cp_emit")


# ---- the compressed cache in decoding, held in 4 bits: thin wrappers, see include/slkv.h ------------------------------------
def slkv_q4_record_bytes(head_dim: int) -> int:
    return int(lib().slkv_q4_record_bytes(int(head_dim)))


def make_q4_cache(records: torch.Tensor, pos: torch.Tensor, weight: Optional[torch.Tensor], starts: torch.Tensor,
                  lens: torch.Tensor, n_kv_heads: int) -> SlkvQ4Cache:
    """records uint8 [slots, slkv_q4_record_bytes], pos int32 [slots], weight float32 [slots] or None, starts int32 [n_seg + 1],
    lens int32 [n_seg], all contiguous.  The structure keeps the tensors alive and belongs to their device."""
    head_dim = {80: 64, 160: 128}[records.size(1)]
    assert records.dtype == torch.uint8 and pos.dtype == starts.dtype == lens.dtype == torch.int32
    assert weight is None or weight.dtype == torch.float32
    tensors = [t for t in (records, pos, weight, starts, lens) if t is not None]
    for t in tensors:
        assert t.is_contiguous() and t.device == records.device and t.dim() == (2 if t is records else 1)
    rows, n_seg = records.size(0), lens.numel()
    assert pos.numel() == rows and (weight is None or weight.numel() == rows) and starts.numel() == n_seg + 1
    assert n_kv_heads >= 1 and n_seg % n_kv_heads == 0
    c = SlkvQ4Cache(n_seg // n_kv_heads, n_kv_heads, head_dim, 0, rows, records.data_ptr(), pos.data_ptr(),
                    weight.data_ptr() if weight is not None else None, starts.data_ptr(), lens.data_ptr())
    c.tensors, c.device, c.lens_tensor = tensors, records.device, lens
    c.index = records.get_device() if records.is_cuda else -2           # no tensor is on that one
    return c


# The calls of a decode step are issued at the rate that the checks below allow: each looks at a property once.  Calls are enqueued
# on a stream of the current device: that has to be the cache's and the tensors'.
_I32, _F32 = torch.int32, torch.float32
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _q4_elsewhere() -> None:
    raise AssertionError("the cache and the tensors have to be on the current device")


def _q4_status(cache: SlkvQ4Cache, status: torch.Tensor) -> None:
    if status.get_device() != cache.index:
        _q4_elsewhere()
    assert status.dtype is _I32 and status.numel() >= 1


def slkv_q4_pack(cache: SlkvQ4Cache, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, kept_idx: torch.Tensor,
                 status: Optional[torch.Tensor] = None, stream=None) -> None:
    """k, v [rows, head_dim], offsets, kept_idx: as slkv_compress wrote them, or slkv_compress_overlapped on the same stream (what is
    queued there goes out first; rows from another stream need a slkv_join)."""
    if not cache.index == k.get_device() == v.get_device() == offsets.get_device() == kept_idx.get_device() == _current_device():
        _q4_elsewhere()
    shape = rows, dim = k.shape
    assert dim == cache.head_dim and v.shape == shape and k.dtype is v.dtype and k.is_contiguous() and v.is_contiguous()
    assert offsets.dtype is _I32 and offsets.is_contiguous() and offsets.numel() == cache.n_seqs * cache.n_kv_heads + 1
    assert kept_idx.dtype is _I32 and kept_idx.is_contiguous() and kept_idx.numel() >= rows
    if status is not None:
        _q4_status(cache, status)
    rc = _fn["slkv_q4_pack"](stream, cache, _DTYPES[k.dtype], k, v, rows, offsets, kept_idx, status)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_q4_pack")


def slkv_q4_append(cache: SlkvQ4Cache, k: torch.Tensor, v: torch.Tensor, pos: torch.Tensor, after: Optional[SlkvQ4Cache] = None,
                   status: Optional[torch.Tensor] = None, stream=None) -> None:
    """k, v [n_seqs, n_tokens, n_kv_heads, head_dim] (any strides over a contiguous last dimension), pos int32 [n_seqs, n_tokens].
    after: the same cache with lengths of its own, which take the new ones."""
    if not cache.index == k.get_device() == v.get_device() == pos.get_device() == _current_device():
        _q4_elsewhere()
    shape = ns, n, hkv, dim = k.shape
    assert ns == cache.n_seqs and hkv == cache.n_kv_heads and dim == cache.head_dim and v.shape == shape and k.dtype is v.dtype
    assert pos.dtype is _I32 and pos.is_contiguous() and pos.numel() == ns * n
    ks, kt, kh, k1 = k.stride()
    vs, vt, vh, v1 = v.stride()
    assert k1 == v1 == 1
    lens_out = None
    if after is not None:
        assert after.records == cache.records and after.starts == cache.starts and after.pos == cache.pos
        assert after.n_seqs == ns and after.n_kv_heads == hkv
        lens_out = after.lens_tensor
    if status is not None:
        _q4_status(cache, status)
    rc = _fn["slkv_q4_append"](stream, cache, _DTYPES[k.dtype], k, v, n, ks, kt, kh, vs, vt, vh, pos, lens_out, status)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_q4_append")


def slkv_q4_unpack(cache: SlkvQ4Cache, k_out: torch.Tensor, v_out: torch.Tensor, slots: Optional[torch.Tensor] = None,
                   stream=None) -> None:
    """k_out, v_out [n, head_dim]: the rows of the slots given (int32 [n], entries outside the cache are padding), or of every
    filled slot at its own place (n = slots of the cache)."""
    if not cache.index == k_out.get_device() == v_out.get_device() == _current_device():
        _q4_elsewhere()
    shape = n, dim = k_out.shape
    assert dim == cache.head_dim and v_out.shape == shape and k_out.dtype is v_out.dtype
    assert k_out.is_contiguous() and v_out.is_contiguous()
    if slots is None:
        assert n == cache.capacity_rows
    else:
        assert slots.dtype is _I32 and slots.is_contiguous() and slots.numel() == n and slots.get_device() == cache.index
        if n == 0:                                         # an empty tensor's address is null, which asks for every slot
            return
    rc = _fn["slkv_q4_unpack"](stream, cache, _DTYPES[k_out.dtype], slots, n, k_out, v_out)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_q4_unpack")


def make_q4_attend(cache: SlkvQ4Cache, q: torch.Tensor, out: torch.Tensor, scale: Optional[float] = None, softcap: float = 0.0,
                   weight_decay: float = 1.0, lse_units: int = SLKV_LSE_LN) -> SlkvQ4AttendParams:
    """Shapes and strides from the tensors: q, out [n_seqs, n_tokens, n_q_heads, head_dim] (last dim contiguous)."""
    assert q.shape == out.shape and q.dim() == 4 and q.dtype == out.dtype and q.stride(3) == 1 and out.stride(3) == 1
    assert q.size(0) == cache.n_seqs and q.size(3) == cache.head_dim
    p = SlkvQ4AttendParams(q.size(2), q.size(1), _DTYPES[q.dtype], lse_units, cache.head_dim ** -0.5 if scale is None else scale,
                           softcap, weight_decay, 0, *q.stride()[:3], *out.stride()[:3])
    p.q_like, p.out_like = (q.shape, q.stride(), q.dtype), (out.shape, out.stride(), out.dtype)
    return p


def slkv_q4_attend_workspace_bytes(cache: SlkvQ4Cache, params: SlkvQ4AttendParams, accumulate: bool = False) -> int:
    return int(lib().slkv_q4_attend_workspace_bytes(C.byref(cache), C.byref(params), int(accumulate)))


def new_q4_workspace(cache: SlkvQ4Cache, params: SlkvQ4AttendParams, accumulate: bool = False) -> torch.Tensor:
    n = slkv_q4_attend_workspace_bytes(cache, params, accumulate)
    if n == 0:
        raise SlkvError(ERR["BAD_SHAPE"], "slkv_q4_attend_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=cache.device)


def slkv_q4_attend(cache: SlkvQ4Cache, params: SlkvQ4AttendParams, q: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                   q_pos: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                   accumulate: bool = False, status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """q, out: the shapes and strides params was made from.  q_pos int32 [n_seqs, n_tokens], slopes float32 [n_q_heads],
    lse float32 [n_seqs, n_q_heads, n_tokens]; accumulate adds to the cache's weights."""
    d = cache.index
    if not d == q.get_device() == out.get_device() == workspace.get_device() == _current_device():
        _q4_elsewhere()
    assert (q.shape, q.stride(), q.dtype) == params.q_like and (out.shape, out.stride(), out.dtype) == params.out_like
    ns, nt, hq, dim = params.q_like[0]
    assert ns == cache.n_seqs and dim == cache.head_dim
    if q_pos is not None:
        assert q_pos.dtype is _I32 and q_pos.is_contiguous() and q_pos.numel() == ns * nt and q_pos.get_device() == d
    if slopes is not None:
        assert slopes.dtype is _F32 and slopes.is_contiguous() and slopes.numel() == hq and slopes.get_device() == d
    if lse is not None:
        assert lse.dtype is _F32 and lse.is_contiguous() and lse.numel() == ns * nt * hq and lse.get_device() == d
    if status is not None:
        _q4_status(cache, status)
    rc = _fn["slkv_q4_attend"](stream, cache, params, q, q_pos, slopes, out, lse, 1 if accumulate else 0, status, workspace,
                               workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_q4_attend")
    return out


def slkv_q4_evict_workspace_bytes(cache: SlkvQ4Cache) -> int:
    return int(lib().slkv_q4_evict_workspace_bytes(C.byref(cache)))


def new_q4_evict_workspace(cache: SlkvQ4Cache, to: Optional[SlkvQ4Cache] = None) -> torch.Tensor:
    """For evictions from `cache` (to whichever cache)."""
    n = slkv_q4_evict_workspace_bytes(cache)
    if n == 0:
        raise SlkvError(ERR["BAD_SHAPE"], "slkv_q4_evict_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=cache.device)


def slkv_q4_evict(cache: SlkvQ4Cache, to: SlkvQ4Cache, budgets: torch.Tensor, window: int, newest: torch.Tensor,
                  workspace: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """budgets int32 [n_kv_heads], newest int32 [n_seqs]; to: `cache` itself, or another cache."""
    if not cache.index == to.index == budgets.get_device() == newest.get_device() == workspace.get_device() == _current_device():
        _q4_elsewhere()
    assert budgets.dtype is _I32 and budgets.is_contiguous() and budgets.numel() == cache.n_kv_heads
    assert newest.dtype is _I32 and newest.is_contiguous() and newest.numel() == cache.n_seqs
    if status is not None:
        _q4_status(cache, status)
    rc = _fn["slkv_q4_evict"](stream, cache, to, budgets, int(window), newest, status, workspace, workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_q4_evict")


# ---- prompts and the paged cache: thin wrappers, see include/slkv.h ----------------------------------------------------------
def make_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, n_seqs: int, window: int = 1,
                scale: Optional[float] = None, lse_units: int = SLKV_LSE_LN) -> SlkvPromptParams:
    """Shapes and strides from the tensors: q, out [tokens, n_q_heads, head_dim], k, v [keys, n_kv_heads, head_dim] (last dim
    contiguous).  window: rows of lse."""
    assert q.dim() == k.dim() == 3 and q.shape == out.shape and k.shape == v.shape and q.size(2) == k.size(2)
    assert q.dtype == k.dtype == v.dtype == out.dtype and q.stride(2) == k.stride(2) == v.stride(2) == out.stride(2) == 1
    p = SlkvPromptParams(n_seqs, q.size(1), k.size(1), q.size(2), window, _DTYPES[q.dtype], lse_units,
                         q.size(2) ** -0.5 if scale is None else scale, *q.stride()[:2], *k.stride()[:2], *v.stride()[:2],
                         *out.stride()[:2])
    p.q_like, p.out_like = (q.shape, q.stride(), q.dtype), (out.shape, out.stride(), out.dtype)
    p.k_like, p.v_like, p.device = (k.shape, k.stride(), k.dtype), (v.shape, v.stride(), v.dtype), q.device
    return p


def _like(t: torch.Tensor):
    return t.shape, t.stride(), t.dtype


def slkv_prompt_attend_workspace_bytes(params: SlkvPromptParams, cu_q: Sequence[int], cu_k: Optional[Sequence[int]] = None) -> int:
    assert len(cu_q) == params.n_seqs + 1 and (cu_k is None or len(cu_k) == len(cu_q))
    return int(lib().slkv_prompt_attend_workspace_bytes(C.byref(params), _cu_host(cu_q), None if cu_k is None else _cu_host(cu_k)))


def new_prompt_workspace(params: SlkvPromptParams, cu_q: Sequence[int], cu_k: Optional[Sequence[int]] = None) -> torch.Tensor:
    n = slkv_prompt_attend_workspace_bytes(params, cu_q, cu_k)
    if n == 0:
        raise SlkvError(ERR["BAD_SHAPE"], "slkv_prompt_attend_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=params.device)


def slkv_prompt_attend(params: SlkvPromptParams, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor,
                       cu_q_host: Sequence[int], out: torch.Tensor, workspace: torch.Tensor, cu_k: Optional[torch.Tensor] = None,
                       cu_k_host: Optional[Sequence[int]] = None, lse: Optional[torch.Tensor] = None,
                       status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """q, k, v, out: the shapes and strides params was made from; cu_q, cu_k int32 [n_seqs + 1] on the device, the same on the host.
    lse float32 [n_seqs, n_q_heads, window]."""
    d = q.get_device()
    if not d == k.get_device() == v.get_device() == cu_q.get_device() == out.get_device() == workspace.get_device() == _current_device():
        _q4_elsewhere()
    assert _like(q) == params.q_like and _like(out) == params.out_like and _like(k) == params.k_like and _like(v) == params.v_like
    n = params.n_seqs
    assert len(cu_q_host) == n + 1 and cu_q.dtype is _I32 and cu_q.is_contiguous() and cu_q.numel() == n + 1
    assert (cu_k is None) == (cu_k_host is None)
    if cu_k is not None:
        assert len(cu_k_host) == n + 1 and cu_k.dtype is _I32 and cu_k.is_contiguous() and cu_k.numel() == n + 1 and cu_k.get_device() == d
    assert cu_q_host[n] <= q.size(0) and (cu_q_host if cu_k is None else cu_k_host)[n] <= k.size(0)
    if lse is not None:
        assert lse.dtype is _F32 and lse.is_contiguous() and lse.get_device() == d
        assert lse.numel() == n * params.n_q_heads * params.window
    if status is not None:
        assert status.dtype is _I32 and status.numel() >= 1 and status.get_device() == d
    rc = _fn["slkv_prompt_attend"](stream, params, q, k, v, cu_q, _cu_list(cu_q_host), cu_k,
                                   None if cu_k is None else _cu_list(cu_k_host), out, lse, status, workspace, workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_prompt_attend")
    return out


def make_paged_cache(k_pages: torch.Tensor, v_pages: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, free_pages: torch.Tensor,
                     n_free: torch.Tensor, n_seqs: int, n_kv_heads: int) -> SlkvPagedCache:
    """k_pages, v_pages [n_pages, page_rows, head_dim], tables int32 [n_segments, max_pages], lens int32 [n_segments], free_pages
    int32 [n_pages], n_free int32 [1], all contiguous; n_segments = layers * n_seqs * n_kv_heads.  The structure keeps the tensors alive
    and belongs to their device."""
    tensors = (k_pages, v_pages, tables, lens, free_pages, n_free)
    assert k_pages.dim() == 3 and k_pages.shape == v_pages.shape and k_pages.dtype == v_pages.dtype
    for t in tensors:
        assert t.is_contiguous() and t.device == k_pages.device
    for t in tensors[2:]:
        assert t.dtype == torch.int32
    n_pages, page_rows, dim = k_pages.shape
    assert tables.dim() == 2 and lens.numel() == tables.size(0) and free_pages.numel() == n_pages and n_free.numel() == 1
    assert n_seqs >= 1 and n_kv_heads >= 1 and lens.numel() % (n_seqs * n_kv_heads) == 0
    c = SlkvPagedCache(lens.numel() // (n_seqs * n_kv_heads), n_seqs, n_kv_heads, dim, _DTYPES[k_pages.dtype], page_rows, n_pages,
                       tables.size(1), *(t.data_ptr() for t in tensors))
    c.tensors, c.device, c.element, c.dim = tensors, k_pages.device, k_pages.dtype, dim
    c.index = k_pages.get_device() if k_pages.is_cuda else -2
    # what calls check, once for all: fields of the structure are slow to read
    c.wanted = (lens.numel(), lens.numel() + c.n_layers, n_seqs)       # by mode of slkv_paged_plan
    c.same = (c.tables, c.free_pages, c.n_layers, n_seqs, n_kv_heads, c.max_pages)
    return c


def slkv_paged_plan(cache: SlkvPagedCache, mode: int, want: torch.Tensor, slots: Optional[torch.Tensor] = None,
                    slot_offsets: Optional[torch.Tensor] = None, after: Optional[SlkvPagedCache] = None,
                    status: Optional[torch.Tensor] = None, stream=None) -> None:
    """want int32: [n_segments] (SLKV_PAGED_LENGTHS), [n_layers, n_seqs * n_kv_heads + 1] (SLKV_PAGED_OFFSETS) or [n_seqs]
    (SLKV_PAGED_ADD).  slots int32: [n] with slot_offsets int32 [n_segments + 1], or [n_segments, width] without (width 0: as no slots).  after: the same cache
    with lengths and a count of free pages of its own, which take the new ones."""
    d = cache.index
    if not d == want.get_device() == _current_device():
        _q4_elsewhere()
    n_seg = cache.wanted[SLKV_PAGED_LENGTHS]
    assert want.dtype is _I32 and want.is_contiguous() and 0 <= mode <= 2 and want.numel() == cache.wanted[mode]
    width = n_slots = 0
    if slots is not None:
        assert slots.dtype is _I32 and slots.is_contiguous() and slots.get_device() == d
        n_slots = slots.numel()
        if slot_offsets is None:
            assert slots.dim() == 2 and slots.size(0) == n_seg
            width = slots.size(1)
            if width == 0:
                slots = None
        else:
            assert slot_offsets.dtype is _I32 and slot_offsets.is_contiguous() and slot_offsets.numel() == n_seg + 1
            assert slot_offsets.get_device() == d
            if n_slots == 0:                     # an empty tensor has no address, which says that no slots are asked for; none is written
                slots = slot_offsets
    lens_out = n_free_out = None
    if after is not None:
        assert after.same == cache.same
        lens_out, n_free_out = after.tensors[3], after.tensors[5]
    if status is not None:
        _q4_status(cache, status)
    rc = _fn["slkv_paged_plan"](stream, cache, mode, want, slots, n_slots, width, slot_offsets, lens_out, n_free_out, status)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_paged_plan")


def slkv_paged_write(cache: SlkvPagedCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, take: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """k, v [n_seqs, n_tokens, n_heads, head_dim] (any strides over a contiguous last dimension) with slots int32 of n_seqs * n_heads *
    width entries and take int32 [n_seqs, width], or [rows, head_dim] with slots int32 [n]."""
    d = cache.index
    if not d == k.get_device() == v.get_device() == slots.get_device() == _current_device():
        _q4_elsewhere()
    assert k.shape == v.shape and k.dtype is v.dtype is cache.element and slots.dtype is _I32 and slots.is_contiguous()
    if k.dim() == 2:
        (nt, dim), ns, hkv = k.shape, 1, 1
        (kt, k1), (vt, v1) = k.stride(), v.stride()
        ks = kh = vs = vh = dim
    else:
        ns, nt, hkv, dim = k.shape
        ks, kt, kh, k1 = k.stride()
        vs, vt, vh, v1 = v.stride()
    assert k1 == v1 == 1 and dim == cache.dim and ns * hkv > 0
    width, rest = divmod(slots.numel(), ns * hkv)
    assert rest == 0
    if take is not None:
        assert take.dtype is _I32 and take.is_contiguous() and take.numel() == ns * width and take.get_device() == d
    rc = _fn["slkv_paged_write"](stream, cache, k, v, ns, hkv, nt, ks, kt, kh, vs, vt, vh, slots, width, take)
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_paged_write")


def make_paged_attend(cache: SlkvPagedCache, q: torch.Tensor, out: torch.Tensor, k_new: Optional[torch.Tensor] = None,
                      v_new: Optional[torch.Tensor] = None, layer: int = 0, scale: Optional[float] = None,
                      lse_units: int = SLKV_LSE_LN) -> SlkvPagedAttendParams:
    """Shapes and strides from the tensors: q, out [n_seqs, n_tokens, n_q_heads, head_dim], k_new, v_new [n_seqs, n_tokens, n_kv_heads,
    head_dim] (last dim contiguous)."""
    assert q.shape == out.shape and q.dim() == 4 and q.dtype == out.dtype == cache.element and q.stride(3) == 1 and out.stride(3) == 1
    assert q.size(0) == cache.n_seqs and q.size(3) == cache.head_dim and (k_new is None) == (v_new is None)
    kv = [(0, 0, 0)] * 2
    if k_new is not None:
        for t in (k_new, v_new):
            assert t.shape == (cache.n_seqs, q.size(1), cache.n_kv_heads, cache.head_dim) and t.dtype == q.dtype and t.stride(3) == 1
        kv = [k_new.stride()[:3], v_new.stride()[:3]]
    p = SlkvPagedAttendParams(q.size(2), q.size(1), layer, int(k_new is not None), lse_units,
                              cache.head_dim ** -0.5 if scale is None else scale, *q.stride()[:3], *out.stride()[:3], *kv[0], *kv[1])
    p.q_like, p.out_like = _like(q), _like(out)
    p.k_like, p.v_like = (None, None) if k_new is None else (_like(k_new), _like(v_new))
    return p


def slkv_paged_attend_workspace_bytes(cache: SlkvPagedCache, params: SlkvPagedAttendParams) -> int:
    return int(lib().slkv_paged_attend_workspace_bytes(C.byref(cache), C.byref(params)))


def new_paged_workspace(cache: SlkvPagedCache, params: SlkvPagedAttendParams) -> torch.Tensor:
    n = slkv_paged_attend_workspace_bytes(cache, params)
    if n == 0:
        raise SlkvError(ERR["BAD_SHAPE"], "slkv_paged_attend_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=cache.device)


def slkv_paged_attend(cache: SlkvPagedCache, params: SlkvPagedAttendParams, q: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                      k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None, tree: Optional[torch.Tensor] = None,
                      n_new: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """q, out, k_new, v_new: the shapes and strides params was made from.  tree int64 (or uint64) [n_seqs, n_tokens], n_new int32 [n_seqs],
    lse float32 [n_seqs, n_q_heads, n_tokens]."""
    d = cache.index
    if not d == q.get_device() == out.get_device() == workspace.get_device() == _current_device():
        _q4_elsewhere()
    assert _like(q) == params.q_like and _like(out) == params.out_like
    ns, nt, hq, dim = params.q_like[0]
    assert ns == cache.n_seqs and dim == cache.head_dim and q.dtype is cache.element
    if params.k_like is None:
        assert k_new is None and v_new is None
    else:
        assert _like(k_new) == params.k_like and _like(v_new) == params.v_like
        assert k_new.get_device() == v_new.get_device() == d and params.k_like[0][2] == cache.n_kv_heads
    if tree is not None:
        assert tree.element_size() == 8 and not tree.is_floating_point() and tree.is_contiguous() and tree.numel() == ns * nt
        assert tree.get_device() == d
    if n_new is not None:
        assert n_new.dtype is _I32 and n_new.is_contiguous() and n_new.numel() == ns and n_new.get_device() == d
    if lse is not None:
        assert lse.dtype is _F32 and lse.is_contiguous() and lse.numel() == ns * nt * hq and lse.get_device() == d
    if status is not None:
        _q4_status(cache, status)
    rc = _fn["slkv_paged_attend"](stream, cache, params, q, k_new, v_new, tree, n_new, out, lse, status, workspace, workspace.numel())
    if rc != SLKV_OK:
        raise SlkvError(rc, "slkv_paged_attend")
    return out
