"""Thin ctypes binding of libilre's C ABI (include/ilre.h).

Argument marshalling only: every step of the recall path runs in the library's HIP kernels.
PyTorch is used for device memory and the current stream, nothing else.  There is no fallback:
if the shared library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libilre.so")

ILRE_OK, ILRE_EINVAL, ILRE_EUNSUPPORTED, ILRE_ENOMEM, ILRE_EHIP = range(5)
ILRE_F32, ILRE_BF16 = 0, 1
ILRE_SCORE_SUM, ILRE_SCORE_MAX = 0, 1
ILRE_FLAG_EXACT_ROW_MAX = 1
ILRE_ROPE_HALF, ILRE_ROPE_INTERLEAVED = 0, 1
ILRE_ROPE_PLAIN, ILRE_ROPE_LINEAR, ILRE_ROPE_BANDS, ILRE_ROPE_PARTS = range(4)
ILRE_MIN_PAGE_TOKENS, ILRE_MAX_PAGE_TOKENS = 16, 32768
ILRE_KV_FP8, ILRE_KV_FP4 = 1, 2
ILRE_KV_BLOCK = 32
ILRE_MAX_AXES = 8
ILRE_MAX_BUDGET = 8192
ILRE_MAX_POOL_KERNEL = 2047
ILRE_MAX_POOL_KERNELS = 64
ILRE_MAX_MAX_KERNEL = 1024
ILRE_MAX_AVG_KERNEL = 1024

ILRE_STATIC_SCRATCH_BYTES = 4 << 20

EXPORTS = ("ilre_workspace_bytes", "ilre_recall", "ilre_row_stats", "ilre_row_stats_static", "ilre_col_scores", "ilre_select",
           "ilre_select_max_avg", "ilre_recall_max_avg", "ilre_workspace_bytes_max_avg", "ilre_rerope_keys",
           "ilre_gather_ids", "ilre_rope_frequencies", "ilre_rope", "ilre_rope_append", "ilre_attention_workspace_bytes",
           "ilre_paged_attention", "ilre_prompt_attention", "ilre_norm_rope", "ilre_norm_rope_append", "ilre_cache_read", "ilre_tree_attention", "ilre_probe_mfma_ceiling", "ilre_probe_describe", "ilre_last_error")


class IlreOpts(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("n_pool_kernels", ctypes.c_int32),
        ("score_mode", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("flags", ctypes.c_int32),
        ("k_stride_head", ctypes.c_int64),
        ("k_stride_token", ctypes.c_int64),
        ("q_stride_head", ctypes.c_int64),
        ("q_stride_token", ctypes.c_int64),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
        ("stream", ctypes.c_void_p),
        ("sink", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


class IlreStrides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("q_token", "q_head", "out_token", "out_head", "k_token", "k_head", "v_token", "v_head")]


class IlrePagedKv(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("page_tokens", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("Hkv", ctypes.c_int32),
        ("stride_page", ctypes.c_int64),
        ("stride_head", ctypes.c_int64),
        ("stride_token", ctypes.c_int64),
        ("k_pages", ctypes.c_void_p),
        ("v_pages", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p),
        ("table_stride", ctypes.c_int64),
        ("kv_len", ctypes.c_void_p),
        ("cu_q", ctypes.c_void_p),
        ("table_width", ctypes.c_int32),
        ("n_seq", ctypes.c_int32),
    ]


class IlreQuantKv(ctypes.Structure):
    _fields_ = [
        ("kv", IlrePagedKv),
        ("format", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("k_scales", ctypes.c_void_p),
        ("v_scales", ctypes.c_void_p),
    ]


class IlreHeadNorms(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("q_norm", ctypes.c_int32),
        ("k_norm", ctypes.c_int32),
        ("offset", ctypes.c_float),
        ("eps", ctypes.c_double),
        ("q_weight", ctypes.c_void_p),
        ("k_weight", ctypes.c_void_p),
    ]


class IlreAttn(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("causal", ctypes.c_int32),
        ("sink", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("max_q", ctypes.c_int32),
        ("max_kv", ctypes.c_int32),
        ("total_kv", ctypes.c_int64),
    ]


class IlreRopeFreqs(ctypes.Structure):
    """A table of rotary frequencies (ilre_rope_frequencies fills one; its fields may be set by hand as well)."""
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("rotary", ctypes.c_int32),
        ("magnitude", ctypes.c_double),
        ("inv_freq", ctypes.c_double * 64),
    ]


class IlreError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"ilre status {status}: {message}")
        self.status = status


_lib = None


def load() -> ctypes.CDLL:
    """Load libilre.so (built in-tree by paper_2508_17892_amd.build); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not built: run `python -m paper_2508_17892_amd.build`")
        lib = ctypes.CDLL(LIB_PATH)
        i64, i32, vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
        po = ctypes.POINTER(IlreOpts)
        lib.ilre_workspace_bytes.restype = ctypes.c_int
        lib.ilre_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        lib.ilre_recall.restype = ctypes.c_int
        lib.ilre_recall.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, ctypes.POINTER(i32), vp, vp, po]
        lib.ilre_row_stats.restype = ctypes.c_int
        lib.ilre_row_stats.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp, vp, po]
        lib.ilre_row_stats_static.restype = ctypes.c_int
        lib.ilre_row_stats_static.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp, vp, po]
        lib.ilre_col_scores.restype = ctypes.c_int
        lib.ilre_col_scores.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp, vp, vp, po]
        lib.ilre_select.restype = ctypes.c_int
        lib.ilre_select.argtypes = [vp, i64, i32, ctypes.POINTER(i32), vp, po]
        pi = ctypes.POINTER(i32)
        lib.ilre_select_max_avg.restype = ctypes.c_int
        lib.ilre_select_max_avg.argtypes = [vp, i64, i32, i32, pi, i32, pi, i32, vp, vp, po]
        lib.ilre_recall_max_avg.restype = ctypes.c_int
        lib.ilre_recall_max_avg.argtypes = [vp, vp, i64, i32, i32, i32, i32, i32, i32, pi, i32, pi, i32, vp, vp, vp, po]
        lib.ilre_workspace_bytes_max_avg.restype = ctypes.c_int
        lib.ilre_workspace_bytes_max_avg.argtypes = [i64, i32, i32, i32, i32, i32, pi, i32, i32, i32,
                                                     ctypes.POINTER(ctypes.c_size_t)]
        lib.ilre_rerope_keys.restype = ctypes.c_int
        lib.ilre_rerope_keys.argtypes = [vp, vp, i64, i32, i32, i32, i32, ctypes.c_double, ctypes.POINTER(ctypes.c_double),
                                         i32, po]
        lib.ilre_gather_ids.restype = ctypes.c_int
        lib.ilre_gather_ids.argtypes = [vp, i64, vp, i32, vp, po]
        ps, pf, pc, pa = (ctypes.POINTER(t) for t in (IlreStrides, IlreRopeFreqs, IlrePagedKv, IlreAttn))
        f64 = ctypes.c_double
        lib.ilre_rope_frequencies.restype = ctypes.c_int
        lib.ilre_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, i32, pf]
        lib.ilre_rope.restype = ctypes.c_int
        lib.ilre_rope.argtypes = [vp, vp, i32, i32, i32, vp, i32, pf, i32, ps, po]
        lib.ilre_rope_append.restype = ctypes.c_int
        lib.ilre_rope_append.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, pf, i32, pc, ps, po]
        lib.ilre_attention_workspace_bytes.restype = ctypes.c_int
        lib.ilre_attention_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32, i32, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
        lib.ilre_paged_attention.restype = ctypes.c_int
        lib.ilre_paged_attention.argtypes = [vp, vp, vp, i32, i32, i32, pa, pc, ps, po]
        lib.ilre_prompt_attention.restype = ctypes.c_int
        lib.ilre_prompt_attention.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, i32, pa, ps, po]
        pn = ctypes.POINTER(IlreHeadNorms)
        lib.ilre_norm_rope.restype = ctypes.c_int
        lib.ilre_norm_rope.argtypes = [vp, vp, i32, i32, i32, vp, i32, vp, i32, pf, i32, pn, ps, po]
        lib.ilre_norm_rope_append.restype = ctypes.c_int
        lib.ilre_norm_rope_append.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, i32, vp, pf, i32, pn, pc, ps, po]
        lib.ilre_cache_read.restype = ctypes.c_int
        lib.ilre_cache_read.argtypes = [vp, vp, i32, i32, vp, pc, ps, po]
        lib.ilre_tree_attention.restype = ctypes.c_int
        lib.ilre_tree_attention.argtypes = [vp, vp, vp, i32, i32, i32, vp, i32, i64, pa, pc, ps, po]
        lib.ilre_probe_mfma_ceiling.restype = ctypes.c_int
        lib.ilre_probe_mfma_ceiling.argtypes = [i32, i32, vp, vp, ctypes.POINTER(ctypes.c_double), po]
        lib.ilre_probe_describe.restype = ctypes.c_char_p
        lib.ilre_probe_describe.argtypes = [i32]
        lib.ilre_last_error.restype = ctypes.c_char_p
        lib.ilre_last_error.argtypes = []
        _lib = lib
    return _lib


def to_device(arr, device="cuda") -> torch.Tensor:
    """Host array (float32, or uint16 holding bf16 bit patterns) -> device tensor of the same bits."""
    import numpy as np
    if arr.dtype == np.uint16:
        return torch.from_numpy(arr.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(arr).to(device)


def ilre_last_error() -> str:
    return load().ilre_last_error().decode()


def _check(rc: int) -> None:
    if rc != ILRE_OK:
        raise IlreError(rc, ilre_last_error())


def ilre_workspace_bytes(L: int, Lq: int, Hq: int, Hkv: int, d: int, n_pool_kernels: int, dtype: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().ilre_workspace_bytes(L, Lq, Hq, Hkv, d, n_pool_kernels, dtype, ctypes.byref(out)))
    return int(out.value)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return ILRE_BF16
    if t.dtype == torch.float32:
        return ILRE_F32
    raise TypeError(f"unsupported element type {t.dtype}")


def _qk_meta(q: torch.Tensor, k: torch.Tensor):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q is [Hq, Lq, d], k_cache is [Hkv, L, d] (any strides with the last dim contiguous)")
    if q.dtype != k.dtype:
        raise TypeError("q and k_cache must share an element type")
    if not (q.is_cuda and k.is_cuda):
        raise ValueError("q and k_cache must be device tensors")
    if q.stride(2) != 1 or k.stride(2) != 1:
        raise ValueError("the head dimension must be contiguous")
    Hq, Lq, d = q.shape
    Hkv, L, d2 = k.shape
    if d != d2:
        raise ValueError("head dims differ")
    return L, Lq, Hq, Hkv, d


def _opts(dtype: int, n_pool_kernels: int, scale: float, score_mode: int, workspace: Optional[torch.Tensor],
          q: Optional[torch.Tensor] = None, k: Optional[torch.Tensor] = None, flags: int = 0, sink: int = 0) -> IlreOpts:
    ks = (0, 0) if k is None else (k.stride(0), k.stride(1))
    qs = (0, 0) if q is None else (q.stride(0), q.stride(1))
    ws = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return IlreOpts(_OPTS_SIZE, dtype, n_pool_kernels, score_mode, float(scale), int(flags), *ks, *qs, *ws, _current_stream(), int(sink), 0)


_OPTS_SIZE = ctypes.sizeof(IlreOpts)


def _current_stream() -> int:
    """Handle of the current stream of the current device (what torch.cuda.current_stream().cuda_stream is, without the stream object)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def alloc_workspace(L: int, Lq: int, Hq: int, Hkv: int, d: int, n_pool_kernels: int, dtype: int,
                    device="cuda") -> torch.Tensor:
    return torch.empty(ilre_workspace_bytes(L, Lq, Hq, Hkv, d, n_pool_kernels, dtype), dtype=torch.uint8, device=device)


def _kernel_array(pool_kernels: Sequence[int]):
    arr = (ctypes.c_int32 * len(pool_kernels))(*[int(w) for w in pool_kernels])
    return arr


def ilre_recall(q: torch.Tensor, k_cache: torch.Tensor, budget: int, pool_kernels: Sequence[int], *,
                scale: float = 0.0, score_mode: int = ILRE_SCORE_SUM, flags: int = 0, sink: int = 0,
                workspace: Optional[torch.Tensor] = None,
                out_idx: Optional[torch.Tensor] = None, out_scores: Optional[torch.Tensor] = None
                ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Whole path; returns (out_idx int32[sink + min(budget, L - sink)] ascending, out_scores float32[L])."""
    L, Lq, Hq, Hkv, d = _qk_meta(q, k_cache)
    dt = _dtype_code(q)
    n = len(pool_kernels)
    if workspace is None:
        workspace = alloc_workspace(L, Lq, Hq, Hkv, d, n, dt, q.device)
    if out_idx is None:
        out_idx = torch.empty(int(sink) + min(int(budget), L - int(sink)), dtype=torch.int32, device=q.device)
    if out_scores is None:
        out_scores = torch.empty(L, dtype=torch.float32, device=q.device)
    o = _opts(dt, n, scale, score_mode, workspace, q, k_cache, flags, sink)
    _check(load().ilre_recall(q.data_ptr(), k_cache.data_ptr(), L, Lq, Hq, Hkv, d, int(budget), _kernel_array(pool_kernels),
                              out_idx.data_ptr(), out_scores.data_ptr(), ctypes.byref(o)))
    return out_idx, out_scores


def ilre_row_stats(q: torch.Tensor, k_cache: torch.Tensor, *, scale: float = 0.0, flags: int = 0,
                   workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Softmax row reference (the row maximum with ILRE_FLAG_EXACT_ROW_MAX) and sum of exponentials
    against it for every row r = h*Lq + i (float32[Hq*Lq] each)."""
    L, Lq, Hq, Hkv, d = _qk_meta(q, k_cache)
    dt = _dtype_code(q)
    if workspace is None:
        workspace = alloc_workspace(L, Lq, Hq, Hkv, d, 0, dt, q.device)
    row_max = torch.empty(Hq * Lq, dtype=torch.float32, device=q.device)
    row_sumexp = torch.empty(Hq * Lq, dtype=torch.float32, device=q.device)
    o = _opts(dt, 0, scale, ILRE_SCORE_SUM, workspace, q, k_cache, flags)
    _check(load().ilre_row_stats(q.data_ptr(), k_cache.data_ptr(), L, Lq, Hq, Hkv, d, row_max.data_ptr(),
                                 row_sumexp.data_ptr(), ctypes.byref(o)))
    return row_max, row_sumexp


def ilre_row_stats_static(q: torch.Tensor, k_cache: torch.Tensor, row_ref: torch.Tensor, row_sumexp: torch.Tensor, *,
                          scale: float = 0.0, flags: int = 0) -> None:
    """ilre_row_stats into the caller's float32[Hq*Lq] outputs, with the library's built-in scratch buffer:
    this wrapper and the call beneath it allocate nothing."""
    L, Lq, Hq, Hkv, d = _qk_meta(q, k_cache)
    for t in (row_ref, row_sumexp):
        if t.dtype != torch.float32 or t.numel() != Hq * Lq or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("row_ref and row_sumexp must be contiguous float32 device vectors of Hq*Lq entries")
    o = _opts(_dtype_code(q), 0, scale, ILRE_SCORE_SUM, None, q, k_cache, flags)
    _check(load().ilre_row_stats_static(q.data_ptr(), k_cache.data_ptr(), L, Lq, Hq, Hkv, d, row_ref.data_ptr(),
                                        row_sumexp.data_ptr(), ctypes.byref(o)))


def ilre_col_scores(q: torch.Tensor, k_cache: torch.Tensor, row_max: torch.Tensor, row_sumexp: torch.Tensor, *,
                    scale: float = 0.0, score_mode: int = ILRE_SCORE_SUM,
                    workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Per-token score (float32[L]) from the row statistics of ilre_row_stats."""
    L, Lq, Hq, Hkv, d = _qk_meta(q, k_cache)
    dt = _dtype_code(q)
    if row_max.numel() != Hq * Lq or row_sumexp.numel() != Hq * Lq:
        raise ValueError("row statistics must have Hq*Lq entries")
    if row_max.dtype != torch.float32 or row_sumexp.dtype != torch.float32:
        raise TypeError("row statistics must be float32")
    if workspace is None:
        workspace = alloc_workspace(L, Lq, Hq, Hkv, d, 0, dt, q.device)
    out = torch.empty(L, dtype=torch.float32, device=q.device)
    o = _opts(dt, 0, scale, score_mode, workspace, q, k_cache)
    _check(load().ilre_col_scores(q.data_ptr(), k_cache.data_ptr(), L, Lq, Hq, Hkv, d, row_max.contiguous().data_ptr(),
                                  row_sumexp.contiguous().data_ptr(), out.data_ptr(), ctypes.byref(o)))
    return out


def ilre_select(scores: torch.Tensor, budget: int, pool_kernels: Sequence[int], *, sink: int = 0,
                workspace: Optional[torch.Tensor] = None, out_idx: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Algorithm 1 on a float32 score vector; returns int32[sink + min(budget, L - sink)] ascending."""
    if scores.dtype != torch.float32 or scores.dim() != 1 or not scores.is_contiguous() or not scores.is_cuda:
        raise ValueError("scores must be a contiguous float32 device vector")
    L = scores.numel()
    n = len(pool_kernels)
    if workspace is None:
        # the selection region is the tail of the full workspace; sized on its own here
        workspace = alloc_workspace(L, 1, 1, 1, 128, n, ILRE_F32, scores.device)
    if out_idx is None:
        out_idx = torch.empty(int(sink) + min(int(budget), L - int(sink)), dtype=torch.int32, device=scores.device)
    o = _opts(ILRE_F32, n, 0.0, ILRE_SCORE_SUM, workspace, sink=sink)
    _check(load().ilre_select(scores.data_ptr(), L, int(budget), _kernel_array(pool_kernels), out_idx.data_ptr(),
                              ctypes.byref(o)))
    return out_idx


def ilre_workspace_bytes_max_avg(L: int, Lq: int, Hq: int, Hkv: int, d: int, sink: int, max_kernels: Sequence[int],
                                 n_avg: int, dtype: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().ilre_workspace_bytes_max_avg(L, Lq, Hq, Hkv, d, int(sink), _kernel_array(max_kernels), len(max_kernels),
                                               int(n_avg), dtype, ctypes.byref(out)))
    return int(out.value)


def alloc_workspace_max_avg(L: int, Lq: int, Hq: int, Hkv: int, d: int, sink: int, max_kernels: Sequence[int], n_avg: int,
                            dtype: int, device="cuda") -> torch.Tensor:
    return torch.empty(ilre_workspace_bytes_max_avg(L, Lq, Hq, Hkv, d, sink, max_kernels, n_avg, dtype), dtype=torch.uint8,
                       device=device)


def ilre_select_max_avg(scores: torch.Tensor, budget: int, max_kernels: Sequence[int], avg_kernels: Sequence[int],
                        sink: int = 0, *, workspace: Optional[torch.Tensor] = None, out_idx: Optional[torch.Tensor] = None,
                        out_count: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Algorithm 1 as printed on a float32 score vector; returns (out_idx int32[sink + min(budget, L - sink)] with
    -1 in unused slots, out_count int32[1])."""
    if scores.dtype != torch.float32 or scores.dim() != 1 or not scores.is_contiguous() or not scores.is_cuda:
        raise ValueError("scores must be a contiguous float32 device vector")
    L = scores.numel()
    if workspace is None:
        workspace = alloc_workspace_max_avg(L, 1, 1, 1, 128, sink, max_kernels, len(avg_kernels), ILRE_F32, scores.device)
    if out_idx is None:
        out_idx = torch.empty(int(sink) + min(int(budget), L - int(sink)), dtype=torch.int32, device=scores.device)
    if out_count is None:
        out_count = torch.empty(1, dtype=torch.int32, device=scores.device)
    o = _opts(ILRE_F32, 0, 0.0, ILRE_SCORE_SUM, workspace)
    _check(load().ilre_select_max_avg(scores.data_ptr(), L, int(sink), int(budget), _kernel_array(max_kernels),
                                      len(max_kernels), _kernel_array(avg_kernels), len(avg_kernels), out_idx.data_ptr(),
                                      out_count.data_ptr(), ctypes.byref(o)))
    return out_idx, out_count


def ilre_recall_max_avg(q: torch.Tensor, k_cache: torch.Tensor, budget: int, max_kernels: Sequence[int],
                        avg_kernels: Sequence[int], sink: int = 0, *, scale: float = 0.0,
                        score_mode: int = ILRE_SCORE_SUM, flags: int = 0, workspace: Optional[torch.Tensor] = None,
                        out_idx: Optional[torch.Tensor] = None, out_count: Optional[torch.Tensor] = None,
                        out_scores: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Whole path with Algorithm 1 as printed; returns (out_idx, out_count, out_scores float32[L])."""
    L, Lq, Hq, Hkv, d = _qk_meta(q, k_cache)
    dt = _dtype_code(q)
    if workspace is None:
        workspace = alloc_workspace_max_avg(L, Lq, Hq, Hkv, d, sink, max_kernels, len(avg_kernels), dt, q.device)
    if out_idx is None:
        out_idx = torch.empty(int(sink) + min(int(budget), L - int(sink)), dtype=torch.int32, device=q.device)
    if out_count is None:
        out_count = torch.empty(1, dtype=torch.int32, device=q.device)
    if out_scores is None:
        out_scores = torch.empty(L, dtype=torch.float32, device=q.device)
    o = _opts(dt, 0, scale, score_mode, workspace, q, k_cache, flags)
    _check(load().ilre_recall_max_avg(q.data_ptr(), k_cache.data_ptr(), L, Lq, Hq, Hkv, d, int(sink), int(budget),
                                      _kernel_array(max_kernels), len(max_kernels), _kernel_array(avg_kernels),
                                      len(avg_kernels), out_idx.data_ptr(), out_count.data_ptr(), out_scores.data_ptr(),
                                      ctypes.byref(o)))
    return out_idx, out_count, out_scores


def ilre_rerope_keys(k_cache: torch.Tensor, chunk_tokens: int, first_extra: int = 0, *, rope_base: float = 10000.0,
                     inv_freq: Optional[Sequence[float]] = None, pairing: int = ILRE_ROPE_HALF,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """DCA re-RoPE of a key cache [Hkv, L, d]; `out` may be k_cache itself (in place) and must share its strides."""
    if k_cache.dim() != 3 or not k_cache.is_cuda or k_cache.stride(2) != 1:
        raise ValueError("k_cache is a device tensor [Hkv, L, d] with the head dimension contiguous")
    Hkv, L, d = k_cache.shape
    if out is None:
        out = torch.empty_strided(k_cache.shape, k_cache.stride(), dtype=k_cache.dtype, device=k_cache.device)
    if out.shape != k_cache.shape or out.stride() != k_cache.stride() or out.dtype != k_cache.dtype:
        raise ValueError("out must have the shape, strides and element type of k_cache")
    o = _opts(_dtype_code(k_cache), 0, 0.0, ILRE_SCORE_SUM, None, None, k_cache)
    freq = None
    if inv_freq is not None:
        if len(inv_freq) != d // 2:
            raise ValueError("inv_freq must have d/2 entries")
        freq = (ctypes.c_double * (d // 2))(*[float(x) for x in inv_freq])
    _check(load().ilre_rerope_keys(k_cache.data_ptr(), out.data_ptr(), L, Hkv, d, int(chunk_tokens), int(first_extra),
                                   float(rope_base), freq, int(pairing), ctypes.byref(o)))
    return out


def ilre_gather_ids(input_ids: torch.Tensor, idx: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """C[I]: the input IDs (int32 device vector) of an index list; -1 where the list holds -1."""
    if input_ids.dtype != torch.int32 or idx.dtype != torch.int32 or not input_ids.is_contiguous() or not idx.is_contiguous():
        raise ValueError("input_ids and idx must be contiguous int32 device vectors")
    if out is None:
        out = torch.empty_like(idx)
    o = _opts(ILRE_F32, 0, 0.0, ILRE_SCORE_SUM, None)
    _check(load().ilre_gather_ids(input_ids.data_ptr(), input_ids.numel(), idx.data_ptr(), idx.numel(), out.data_ptr(),
                                  ctypes.byref(o)))
    return out


def _tokens_view(name: str, t: torch.Tensor, heads: Optional[int] = None):
    """(tokens, heads, d, token stride, head stride) of a device tensor [tokens, heads, d].  The strides of a lone token or head say nothing (torch may
    hold anything there) and go as 0; 0 stands for contiguous in the C ABI, so that a tensor expanded over tokens or heads has to be refused here."""
    shape = t.shape
    if len(shape) != 3 or not t.is_cuda:
        raise ValueError(f"{name} is a device tensor [tokens, heads, d] with the head dimension contiguous")
    n, h, d = shape
    s0, s1, s2 = t.stride()
    if s2 != 1:
        raise ValueError(f"{name} is a device tensor [tokens, heads, d] with the head dimension contiguous")
    if heads is not None and h != heads:
        raise ValueError(f"{name} has {h} heads, not {heads}")
    if n <= 1:
        s0 = 0
    elif s0 == 0:
        raise ValueError(f"{name}: tensors expanded over tokens or heads are not supported")
    if h <= 1:
        s1 = 0
    elif s1 == 0:
        raise ValueError(f"{name}: tensors expanded over tokens or heads are not supported")
    return n, h, d, s0, s1


def _int32_vector(name: str, t: torch.Tensor, n: int) -> int:
    if t.dtype != torch.int32 or not t.is_cuda or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} is a contiguous int32 device vector of {n} entries")
    return t.data_ptr()


@functools.lru_cache(maxsize=4096)
def _strides_ref(*values: int):
    """An ilre_strides of these values to pass on (the library only reads it)."""
    return ctypes.byref(IlreStrides(*values))


@functools.lru_cache(maxsize=4096)
def _attn_ref(causal: int, sink: int, window: int, max_q: int, max_kv: int, total_kv: int):
    return ctypes.byref(IlreAttn(ctypes.sizeof(IlreAttn), causal, sink, window, max_q, max_kv, total_kv))


@functools.lru_cache(maxsize=4096)
def _call_opts_ref(dtype: int, scale: float, workspace: int, workspace_bytes: int, stream: int):
    """An ilre_opts of the operators around a recall to pass on (the library only reads it)."""
    return ctypes.byref(IlreOpts(_OPTS_SIZE, dtype, 0, ILRE_SCORE_SUM, scale, 0, 0, 0, 0, 0, workspace, workspace_bytes, stream, 0, 0))


def _like(name: str, out: Optional[torch.Tensor], ref: torch.Tensor):
    """(out, its token stride, its head stride): a new tensor, or the caller's of the same shape and element type."""
    if out is None:
        out = torch.empty(ref.shape, dtype=ref.dtype, device=ref.device)
    elif out.shape != ref.shape or out.dtype != ref.dtype:
        raise ValueError(f"{name} must have the shape and element type of its input")
    return (out, *_tokens_view(name, out)[3:])


def ilre_rope_frequencies(rotary: int, base: float, *, scaling: int = ILRE_ROPE_PLAIN, factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                          original_len: int = 0) -> IlreRopeFreqs:
    """Rotary frequencies (a host table that a program keeps): plain, divided by a factor, or scaled by bands or by parts; see include/ilre.h."""
    f = IlreRopeFreqs()
    _check(load().ilre_rope_frequencies(int(rotary), float(base), int(scaling), float(factor), float(low), float(high), int(original_len), ctypes.byref(f)))
    return f


def ilre_rope(x: torch.Tensor, freqs: IlreRopeFreqs, positions: Optional[torch.Tensor] = None, *, first_position: int = 0,
              pairing: int = ILRE_ROPE_HALF, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotary positions of x [T, H, d]; `out` may be x itself, or a view of the recall's key cache: k_cache[:, a:a+T].transpose(0, 1)."""
    T, H, d, x0, x1 = _tokens_view("x", x)
    out, o0, o1 = _like("out", out, x)
    if T == 0:
        return out
    st = _strides_ref(x0, x1, o0, o1)
    o = _opts(_dtype_code(x), 0, 0.0, ILRE_SCORE_SUM, None)
    _check(load().ilre_rope(x.data_ptr(), out.data_ptr(), T, H, d, None if positions is None else _int32_vector("positions", positions, T),
                            int(first_position), ctypes.byref(freqs), int(pairing), st, ctypes.byref(o)))
    return out


class PagedKV:
    """A cache of pages and the sequences of a call, described once and kept: the tensors are referred to, not copied, and what a program
    writes into page_table, kv_len and cu_q later counts in later calls.

    k_pages, v_pages [num_pages, Hkv, page_tokens, d] in any layout with d contiguous (both the same; v_pages None: keys only),
    page_table int32 [n_seq, pages a sequence], kv_len int32 [n_seq] (new tokens included), cu_q int32 [n_seq + 1]."""

    def __init__(self, k_pages: torch.Tensor, v_pages: Optional[torch.Tensor], page_table: torch.Tensor, kv_len: torch.Tensor, cu_q: torch.Tensor):
        if k_pages.dim() != 4 or not k_pages.is_cuda or k_pages.stride(3) != 1:
            raise ValueError("k_pages is a device tensor [num_pages, Hkv, page_tokens, d] with the head dimension contiguous")
        if v_pages is not None and (v_pages.shape != k_pages.shape or v_pages.stride() != k_pages.stride() or v_pages.dtype != k_pages.dtype
                                    or not v_pages.is_cuda):
            raise ValueError("v_pages must have the shape, strides and element type of k_pages")
        if any(s == 0 and n > 1 for s, n in zip(k_pages.stride(), k_pages.shape)):
            raise ValueError("pages expanded over a dimension are not supported")
        self.dtype = _dtype_code(k_pages)
        c = IlrePagedKv()
        c.struct_size = ctypes.sizeof(IlrePagedKv)
        self._describe(c, k_pages, v_pages, page_table, kv_len, cu_q, 1)

    def _describe(self, c: IlrePagedKv, k_pages, v_pages, page_table, kv_len, cu_q, per: int) -> None:
        """Fill in c; an element of the pages holds `per` channels."""
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or not page_table.is_cuda or page_table.stride(1) != 1:
            raise ValueError("page_table is an int32 device tensor [n_seq, pages] with contiguous rows")
        n_seq = page_table.shape[0]
        if n_seq > 1 and page_table.stride(0) == 0:  # (0 stands for contiguous in the C ABI)
            raise ValueError("a page_table expanded over sequences is not supported")
        num_pages, Hkv, P, d = k_pages.shape
        d *= per
        if d != 128:
            raise IlreError(ILRE_EUNSUPPORTED, f"head_dim {d} unsupported (only 128)")
        self.k_pages, self.v_pages, self.page_table, self.kv_len, self.cu_q = k_pages, v_pages, page_table, kv_len, cu_q
        self.n_seq, self.Hkv = n_seq, Hkv
        self.c = c
        c.page_tokens, c.num_pages, c.Hkv = P, num_pages, Hkv
        # the strides of a lone page or head say nothing
        c.stride_token = k_pages.stride(2) * per
        c.stride_head = k_pages.stride(1) * per if Hkv > 1 else d
        c.stride_page = k_pages.stride(0) * per if num_pages > 1 else d
        c.k_pages, c.v_pages = k_pages.data_ptr(), 0 if v_pages is None else v_pages.data_ptr()
        c.page_table, c.table_width, c.n_seq = page_table.data_ptr(), page_table.shape[1], n_seq
        c.table_stride = page_table.stride(0) if n_seq > 1 else page_table.shape[1]
        c.kv_len, c.cu_q = _int32_vector("kv_len", kv_len, n_seq), _int32_vector("cu_q", cu_q, n_seq + 1)
        self._ref = ctypes.byref(c)


class QuantKV(PagedKV):
    """A cache of pages held in 8 or 4 bits with a scale for every 32 channels, described once and kept like a PagedKV; every call that takes a PagedKV takes one.

    k_pages, v_pages: codes, float8_e4m3fn [num_pages, Hkv, page_tokens, 128] (8 bits) or uint8 [num_pages, Hkv, page_tokens, 64] (4 bits, channel 2i in the lower half
    of byte i), in any layout of pages, heads and tokens; k_scales, v_scales: uint8 [num_pages, Hkv, page_tokens, 4] in the same layout (a byte b stands for 2^(b - 127));
    v_pages and v_scales None: keys only."""

    def __init__(self, k_pages: torch.Tensor, v_pages: Optional[torch.Tensor], k_scales: torch.Tensor, v_scales: Optional[torch.Tensor], page_table: torch.Tensor,
                 kv_len: torch.Tensor, cu_q: torch.Tensor):
        if k_pages.dtype not in (torch.float8_e4m3fn, torch.uint8):
            raise TypeError(f"unsupported element type {k_pages.dtype}: codes are float8_e4m3fn or (4 bits) uint8")
        fp8 = k_pages.dtype == torch.float8_e4m3fn
        if k_pages.dim() != 4 or not k_pages.is_cuda or k_pages.stride(3) != 1 or k_scales.dim() != 4 or k_scales.stride(3) != 1:
            raise ValueError("k_pages and k_scales are device tensors [num_pages, Hkv, page_tokens, .] with the last dimension contiguous")
        if (v_pages is None) != (v_scales is None):
            raise ValueError("v_pages and v_scales go together")
        if v_pages is not None and (v_pages.shape != k_pages.shape or v_pages.stride() != k_pages.stride() or v_pages.dtype != k_pages.dtype
                                    or not v_pages.is_cuda):
            raise ValueError("v_pages must have the shape, strides and element type of k_pages")
        per, scale = (1, 32) if fp8 else (2, 16)  # channels an element of the pages, elements a scale
        for name, t in (("k_scales", k_scales), ("v_scales", v_scales)):
            if t is None:
                continue
            if t.dtype != torch.uint8 or not t.is_cuda or t.shape != (*k_pages.shape[:3], 4):
                raise ValueError(f"{name} is a uint8 device tensor [num_pages, Hkv, page_tokens, 4]")
            if t.stride(3) != 1 or any(n > 1 and a != b * scale for n, a, b in zip(k_pages.shape[:3], k_pages.stride(), t.stride())):
                raise ValueError(f"{name} must have the layout of the codes (a {scale}th of their strides)")
        if any(s == 0 and n > 1 for s, n in zip(k_pages.stride(), k_pages.shape)):
            raise ValueError("pages expanded over a dimension are not supported")
        if any(t is not None and t.get_device() != k_pages.get_device() for t in (v_pages, k_scales, v_scales, page_table, kv_len, cu_q)):
            raise ValueError("pages, scales, page_table, kv_len and cu_q are on one device")
        self.dtype = None  # of the states: any
        self.k_scales, self.v_scales = k_scales, v_scales
        q = self.quant = IlreQuantKv()
        q.format = ILRE_KV_FP8 if fp8 else ILRE_KV_FP4
        q.k_scales, q.v_scales = k_scales.data_ptr(), 0 if v_scales is None else v_scales.data_ptr()
        c = q.kv
        c.struct_size = ctypes.sizeof(IlreQuantKv)
        self._describe(c, k_pages, v_pages, page_table, kv_len, cu_q, per)


class HeadNorms:
    """Norms of queries and keys for each head, x / sqrt(mean(x^2) + eps) * (weight + offset), described once and kept.  q_weight, k_weight [128] in the states' element
    type; None: that one is not normed."""

    def __init__(self, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor] = None, *, eps: float = 1e-6, offset: float = 0.0):
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            if w is not None and (not w.is_cuda or w.dim() != 1 or w.numel() != 128 or not w.is_contiguous()):
                raise ValueError(f"{name} is a contiguous device vector of 128 entries")
        if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
            raise TypeError("q_weight and k_weight must share an element type")
        self.q_weight, self.k_weight = q_weight, k_weight
        w = q_weight if q_weight is not None else k_weight
        self.dtype = None if w is None else _dtype_code(w)
        self.c = IlreHeadNorms(ctypes.sizeof(IlreHeadNorms), 0 if q_weight is None else 1, 0 if k_weight is None else 1, float(offset), float(eps),
                               None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr())
        self._ref = ctypes.byref(self.c)


def _weights_of(norms: Optional[HeadNorms]):
    return () if norms is None else (norms.q_weight, norms.k_weight)


@functools.lru_cache(maxsize=256)
def _axes_array(axes: Tuple[int, ...]):
    if any(not 0 <= a < 256 for a in axes):
        raise ValueError("axes are numbers of rows of positions")
    return (ctypes.c_uint8 * len(axes))(*axes)


def _turn_arguments(freqs: Optional[IlreRopeFreqs], positions: Optional[torch.Tensor], axes: Optional[Sequence[int]], T: int):
    """(positions, number of axes, axes, frequencies) as the C ABI takes them: positions [T], or [number of axes, T] with `axes`, the axis that each pair turns by."""
    if freqs is None:
        return None, 1, None, None
    if axes is None:
        return None if positions is None else _int32_vector("positions", positions, T), 1, None, ctypes.byref(freqs)
    if len(axes) != freqs.rotary // 2:
        raise ValueError(f"axes has an entry for each of the {freqs.rotary // 2} pairs")
    if positions is None or positions.dtype != torch.int32 or not positions.is_cuda or positions.dim() != 2 or positions.shape[1] != T or not positions.is_contiguous():
        raise ValueError(f"positions is a contiguous int32 device tensor [axes, {T}]")
    return positions.data_ptr(), positions.shape[0], _axes_array(tuple(axes)), ctypes.byref(freqs)


def _stream_of(*tensors: Optional[torch.Tensor]) -> int:
    """The current stream of the current device, on which the library works: a tensor of another device would be reached over the link, or not at all, on a stream that does not wait
    for it, and is refused."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor on device {t.get_device()}, the current device is {here}")
    return torch._C._cuda_getCurrentRawStream(here)


def ilre_rope_append(q: Optional[torch.Tensor], k: torch.Tensor, v: Optional[torch.Tensor], cache: PagedKV, freqs: IlreRopeFreqs,
                     positions: Optional[torch.Tensor] = None, *, pairing: int = ILRE_ROPE_HALF, q_out: Optional[torch.Tensor] = None
                     ) -> Optional[torch.Tensor]:
    """Turn queries (returned, or in q_out, which may be q) and keys to their positions (default: their places in the cache) and store keys and values in
    the cache.  q [T, Hq, d], k and v [T, Hkv, d], any token and head strides; q None: keys and values only; v None: keys only."""
    T, Hq, d, dt, q_out, st = _append_arguments(q, k, v, cache, q_out)
    if T == 0:
        return q_out
    pos = None if positions is None else _int32_vector("positions", positions, T)
    o = _call_opts_ref(dt, 0.0, 0, 0, _stream_of(q, k, v, q_out, positions, cache.k_pages))
    _check(load().ilre_rope_append(None if q is None else q.data_ptr(), None if q is None else q_out.data_ptr(), k.data_ptr(),
                                   None if v is None else v.data_ptr(), T, Hq, d, pos, ctypes.byref(freqs), int(pairing), cache._ref, st, o))
    return q_out


def _append_arguments(q, k, v, cache: PagedKV, q_out):
    """(tokens, query heads, d, element type, q_out, strides) of a call that fills a cache."""
    T, _, d, k0, k1 = _tokens_view("k", k, cache.Hkv)
    dt = _dtype_code(k)
    if cache.dtype not in (dt, None) or (q is not None and q.dtype != k.dtype) or (v is not None and v.dtype != k.dtype):
        raise TypeError("q, k, v and the cache must share an element type")
    q0 = q1 = o0 = o1 = v0 = v1 = 0
    Hq = cache.Hkv
    if q is not None:
        Tq, Hq, dq, q0, q1 = _tokens_view("q", q)
        if Tq != T or dq != d:
            raise ValueError("q and k differ in tokens or head dimension")
        q_out, o0, o1 = _like("q_out", q_out, q)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if v is not None:
        Tv, _, dv, v0, v1 = _tokens_view("v", v, cache.Hkv)
        if Tv != T or dv != d:
            raise ValueError("k and v differ in shape")
        if cache.v_pages is None:
            raise ValueError("the cache holds keys only")
    return T, Hq, d, dt, q_out, _strides_ref(q0, q1, o0, o1, k0, k1, v0, v1)


def ilre_norm_rope(x: torch.Tensor, freqs: Optional[IlreRopeFreqs], positions: Optional[torch.Tensor] = None, *, norms: Optional[HeadNorms] = None,
                   axes: Optional[Sequence[int]] = None, first_position: int = 0, pairing: int = ILRE_ROPE_HALF, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Norm of every head of x [T, H, d] (norms.q_weight) and rotation to its position; freqs None: no rotation; positions [T], or [number of axes, T] with `axes`, the axis
    that each pair turns by; `out` may be x itself."""
    T, H, d, x0, x1 = _tokens_view("x", x)
    dt = _dtype_code(x)
    if norms is not None and norms.dtype not in (dt, None):
        raise TypeError("x and the norms' weights must share an element type")
    out, o0, o1 = _like("out", out, x)
    pos, n_axes, ax, fr = _turn_arguments(freqs, positions, axes, T)
    if T == 0:
        return out
    o = _call_opts_ref(dt, 0.0, 0, 0, _stream_of(x, out, positions, *_weights_of(norms)))
    _check(load().ilre_norm_rope(x.data_ptr(), out.data_ptr(), T, H, d, pos, n_axes, ax, int(first_position), fr, int(pairing),
                                 None if norms is None else norms._ref, _strides_ref(x0, x1, o0, o1), o))
    return out


def ilre_norm_rope_append(q: Optional[torch.Tensor], k: torch.Tensor, v: Optional[torch.Tensor], cache: PagedKV, freqs: Optional[IlreRopeFreqs],
                          positions: Optional[torch.Tensor] = None, *, norms: Optional[HeadNorms] = None, axes: Optional[Sequence[int]] = None,
                          pairing: int = ILRE_ROPE_HALF, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """ilre_rope_append with a norm of every query and key head before the rotation, and with positions along several axes (positions [number of axes, T], axes: the
    axis that each pair turns by); freqs None: no rotation.  The cache may be a QuantKV."""
    T, Hq, d, dt, q_out, st = _append_arguments(q, k, v, cache, q_out)
    if norms is not None and norms.dtype not in (dt, None):
        raise TypeError("the states and the norms' weights must share an element type")
    pos, n_axes, ax, fr = _turn_arguments(freqs, positions, axes, T)
    if T == 0:
        return q_out
    o = _call_opts_ref(dt, 0.0, 0, 0, _stream_of(q, k, v, q_out, positions, cache.k_pages, *_weights_of(norms)))
    _check(load().ilre_norm_rope_append(None if q is None else q.data_ptr(), None if q is None else q_out.data_ptr(), k.data_ptr(),
                                        None if v is None else v.data_ptr(), T, Hq, d, pos, n_axes, ax, fr, int(pairing),
                                        None if norms is None else norms._ref, cache._ref, st, o))
    return q_out


def ilre_cache_read(cache: PagedKV, T: int, tokens: Optional[torch.Tensor] = None, *, dtype: Optional[torch.dtype] = None, values: bool = True,
                    k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Keys and values out of a paged cache, T rows cut up by cache.cu_q: the tokens `tokens` (int32 [T]), or the last tokens of each sequence.  Returns (k_out, v_out) [T,
    Hkv, d]; the caller's own tensors (k_out alone: keys only) may be views of the recall's key cache, k_cache.transpose(0, 1).  dtype: of the rows, bfloat16 (the default) or float32 out of a
    quantised cache; a cache of the states' own type, and the caller's tensors, have theirs."""
    if k_out is None and v_out is None:
        dt = (dtype or torch.bfloat16) if cache.dtype is None else cache.k_pages.dtype
        if dtype not in (dt, None):
            raise TypeError(f"the cache holds {dt}, not {dtype}")
        k_out = torch.empty((T, cache.Hkv, 128), dtype=dt, device=cache.k_pages.device)
        v_out = torch.empty_like(k_out) if values and cache.v_pages is not None else None
    k0 = k1 = v0 = v1 = 0
    ref = k_out if k_out is not None else v_out
    if dtype not in (ref.dtype, None):
        raise TypeError(f"k_out and v_out are {ref.dtype}, not {dtype}")
    dt = _dtype_code(ref)
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is None:
            continue
        n, _, d, s0, s1 = _tokens_view(name, t, cache.Hkv)
        if n != T or d != 128 or t.dtype != ref.dtype:
            raise ValueError(f"{name} is a device tensor [{T}, {cache.Hkv}, 128] of one element type")
        if name == "k_out":
            k0, k1 = s0, s1
        else:
            v0, v1 = s0, s1
    if cache.dtype not in (dt, None):
        raise TypeError("the cache and what is read from it must share an element type")
    if v_out is not None and cache.v_pages is None:
        raise ValueError("the cache holds keys only")
    if T == 0:
        return k_out, v_out
    at = None if tokens is None else _int32_vector("tokens", tokens, T)
    o = _call_opts_ref(dt, 0.0, 0, 0, _stream_of(k_out, v_out, tokens, cache.k_pages))
    _check(load().ilre_cache_read(None if k_out is None else k_out.data_ptr(), None if v_out is None else v_out.data_ptr(), T, 128, at,
                                  cache._ref, _strides_ref(0, 0, 0, 0, k0, k1, v0, v1), o))
    return k_out, v_out


def ilre_attention_workspace_bytes(T: int, n_seq: int, Hq: int, Hkv: int, d: int, max_q: int, max_kv: int, total_kv: int, dtype: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().ilre_attention_workspace_bytes(int(T), int(n_seq), Hq, Hkv, d, int(max_q), int(max_kv), int(total_kv), dtype, ctypes.byref(out)))
    return int(out.value)


def alloc_workspace_attention(T: int, n_seq: int, Hq: int, Hkv: int, d: int, max_q: int, max_kv: int, *, total_kv: int = 0, dtype: int = ILRE_BF16,
                              device="cuda") -> torch.Tensor:
    return torch.empty(ilre_attention_workspace_bytes(T, n_seq, Hq, Hkv, d, max_q, max_kv, total_kv, dtype), dtype=torch.uint8, device=device)


def _attention_outputs(q: torch.Tensor, out: Optional[torch.Tensor], lse: Optional[torch.Tensor], T: int, Hq: int):
    out, o0, o1 = _like("out", out, q)
    if lse is None:
        lse = torch.empty((T, Hq), dtype=torch.float32, device=q.device)
    elif lse.dtype != torch.float32 or lse.shape != (T, Hq) or not lse.is_contiguous() or not lse.is_cuda:
        raise ValueError("lse is a contiguous float32 device tensor [T, Hq]")
    return out, o0, o1, lse


def ilre_paged_attention(q: torch.Tensor, cache: PagedKV, *, max_q: int, max_kv: int, total_kv: int = 0, causal: bool = True, sink: int = 0,
                         window: int = 0, scale: float = 0.0, workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                         lse: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of new tokens q [T, Hq, d] over a paged cache that holds them already; returns (out [T, Hq, d], lse float32 [T, Hq]).
    max_q, max_kv, total_kv: the most new tokens and tokens of a sequence, and all tokens together (0: not known); they decide how the work is
    cut up, not what comes out."""
    T, Hq, d, q0, q1 = _tokens_view("q", q)
    dt = _dtype_code(q)
    if cache.dtype not in (dt, None):
        raise TypeError("q and the cache must share an element type")
    if cache.v_pages is None:
        raise ValueError("the cache holds keys only")
    out, o0, o1, lse = _attention_outputs(q, out, lse, T, Hq)
    if T == 0:
        return out, lse
    if workspace is None:
        workspace = alloc_workspace_attention(T, cache.n_seq, Hq, cache.Hkv, d, max_q, max_kv, total_kv=total_kv, dtype=dt, device=q.device)
    elif not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace is a contiguous device tensor")
    at = _attn_ref(1 if causal else 0, int(sink), int(window), int(max_q), int(max_kv), int(total_kv))
    st = _strides_ref(q0, q1, o0, o1)
    o = _call_opts_ref(dt, float(scale), workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_of(q, out, lse, workspace, cache.k_pages))
    _check(load().ilre_paged_attention(q.data_ptr(), out.data_ptr(), lse.data_ptr(), T, Hq, d, at, cache._ref, st, o))
    return out, lse


def ilre_tree_attention(q: torch.Tensor, cache: PagedKV, tree: torch.Tensor, *, max_q: int, max_kv: int, total_kv: int = 0, scale: float = 0.0,
                        workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None
                        ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of drafted tokens q [T, Hq, d], stored at the ends of their sequences: each sees all of the context before them, and those of its sequence's drafted tokens
    whose bit is set in its row of `tree` (int32 [T, words], bit j % 32 of word j / 32).  Returns (out [T, Hq, d], lse float32 [T, Hq])."""
    T, Hq, d, q0, q1 = _tokens_view("q", q)
    dt = _dtype_code(q)
    if cache.dtype not in (dt, None):
        raise TypeError("q and the cache must share an element type")
    if cache.v_pages is None:
        raise ValueError("the cache holds keys only")
    if tree.dtype != torch.int32 or not tree.is_cuda or tree.dim() != 2 or tree.shape[0] != T or (tree.shape[1] > 1 and tree.stride(1) != 1):
        raise ValueError(f"tree is an int32 device tensor [{T}, words] with contiguous rows")
    words, row = tree.shape[1], tree.stride(0) if T > 1 else 0
    if T > 1 and row == 0:  # (0 stands for contiguous in the C ABI)
        raise ValueError("a tree expanded over tokens is not supported")
    out, o0, o1, lse = _attention_outputs(q, out, lse, T, Hq)
    if T == 0:
        return out, lse
    if workspace is None:
        workspace = alloc_workspace_attention(T, cache.n_seq, Hq, cache.Hkv, d, max_q, max_kv, total_kv=total_kv, dtype=dt, device=q.device)
    elif not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace is a contiguous device tensor")
    at = _attn_ref(0, 0, 0, int(max_q), int(max_kv), int(total_kv))
    o = _call_opts_ref(dt, float(scale), workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_of(q, tree, out, lse, workspace, cache.k_pages))
    _check(load().ilre_tree_attention(q.data_ptr(), out.data_ptr(), lse.data_ptr(), T, Hq, d, tree.data_ptr(), words, row, at, cache._ref,
                                      _strides_ref(q0, q1, o0, o1), o))
    return out, lse


def ilre_prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, *, cu_k: Optional[torch.Tensor] = None, max_q: int,
                          max_k: Optional[int] = None, causal: bool = True, sink: int = 0, window: int = 0, scale: float = 0.0,
                          workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None
                          ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of packed sequences, q [T, Hq, d], k and v [Tk, Hkv, d], cut up by cu_q and cu_k (int32 [n_seq + 1]; cu_k None: cu_q); the last
    queries of a sequence stand at its last keys.  Returns (out [T, Hq, d], lse float32 [T, Hq])."""
    T, Hq, d, q0, q1 = _tokens_view("q", q)
    Tk, Hkv, dk, k0, k1 = _tokens_view("k", k)
    Tv, _, dv, v0, v1 = _tokens_view("v", v, Hkv)
    if Tv != Tk or dv != dk or dk != d:
        raise ValueError("k and v differ in shape, or from q in the head dimension")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k and v must share an element type")
    n_seq = cu_q.numel() - 1
    pq = _int32_vector("cu_q", cu_q, n_seq + 1)
    pk = None if cu_k is None else _int32_vector("cu_k", cu_k, n_seq + 1)
    max_k = max_q if max_k is None else max_k
    dt = _dtype_code(q)
    out, o0, o1, lse = _attention_outputs(q, out, lse, T, Hq)
    if T == 0:
        return out, lse
    if workspace is None:
        workspace = alloc_workspace_attention(T, n_seq, Hq, Hkv, d, max_q, max_k, total_kv=Tk, dtype=dt, device=q.device)
    elif not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace is a contiguous device tensor")
    at = _attn_ref(1 if causal else 0, int(sink), int(window), int(max_q), int(max_k), Tk)
    st = _strides_ref(q0, q1, o0, o1, k0, k1, v0, v1)
    o = _opts(dt, 0, scale, ILRE_SCORE_SUM, workspace)
    _check(load().ilre_prompt_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), T, Tk, Hq, Hkv, d, pq, pk, n_seq, at, st, ctypes.byref(o)))
    return out, lse


ILRE_PROBE_OPERAND_BYTES = 65536
ILRE_PROBE_OUT_BYTES = (1 << 20) + 4096


def ilre_probe_describe(variant: int) -> Optional[str]:
    text = load().ilre_probe_describe(int(variant))
    return text.decode() if text else None


def ilre_probe_mfma_ceiling(variant: int, iters: int, operands: torch.Tensor, out: torch.Tensor) -> float:
    """Enqueue one launch of a register-only MFMA loop (measurement aid); returns the MFMA flops of the launch.
    `out` (uint8, ILRE_PROBE_OUT_BYTES) receives, from byte 1 MiB on, per workgroup (shader cycles, 100 MHz ticks)."""
    if operands.numel() * operands.element_size() < ILRE_PROBE_OPERAND_BYTES or not operands.is_cuda:
        raise ValueError("operands must hold ILRE_PROBE_OPERAND_BYTES on the device")
    if out.numel() * out.element_size() < ILRE_PROBE_OUT_BYTES or not out.is_cuda:
        raise ValueError("out must hold ILRE_PROBE_OUT_BYTES on the device")
    o = _opts(ILRE_BF16, 0, 0.0, ILRE_SCORE_SUM, None)
    flops = ctypes.c_double(0.0)
    _check(load().ilre_probe_mfma_ceiling(int(variant), int(iters), operands.data_ptr(), out.data_ptr(), ctypes.byref(flops),
                                          ctypes.byref(o)))
    return float(flops.value)
