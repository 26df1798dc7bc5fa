"""Thin ctypes binding of ``libspindlekv.so``: same names as the C ABI, argument marshalling only.

Every step of the reduction pass runs in the library's CUDA kernels; torch is used for device
memory and streams.  Loading fails loudly when the library is missing and cannot be built.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
from typing import Optional, Sequence

import numpy as np
import torch

from . import build as _build

OK, INVALID_ARG, BUDGET, WORKSPACE_TOO_SMALL, CAPACITY, UNSUPPORTED, CUDA_ERROR, TIMEOUT = range(8)
F32, BF16 = 0, 1
MODE_EVICT, MODE_CODEBOOK = 1, 2
WS_EVICT, WS_CODEBOOK = 0, 1
PAGED_INT8, PAGED_E4M3 = 0, 1
PAGED_BLOCK = 16
KERNEL_CLASSES = ("window_score", "topk", "norms", "similarity", "degree", "greedy", "finalise", "gather",
                  "similarity_fallback", "decode", "paged_attend", "paged_append", "pages", "beam", "prompt", "logits")


class SpindleKVError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_lib.spindlekv_status_string(status).decode()} (status {status})")


class _Tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32), ("stride_layer", C.c_int64),
                ("stride_seq", C.c_int64), ("stride_head", C.c_int64), ("stride_tok", C.c_int64)]


class _Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("window", C.c_int32), ("n_shallow", C.c_int32),
                ("reserve_ratio", C.c_double), ("budget_tokens", C.c_double), ("beta", C.c_double),
                ("theta_k", C.c_float), ("theta_v", C.c_float), ("score_norm", C.c_int32),
                ("per_query_head", C.c_int32)]


class _Batch(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_seqs", C.c_int32), ("max_len", C.c_int32),
                ("total_len", C.c_int32), ("cu_seqlens", C.c_void_p), ("layer_lens", C.c_void_p), ("layer_lens_heads", C.c_int32)]


class _PagePool(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("page_ref", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("format", C.c_int32)]


class _PageTable(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("lens", C.c_void_p), ("n_layers", C.c_int32), ("n_seqs", C.c_int32), ("max_pages", C.c_int32)]


class _LogitRules(C.Structure):
    _fields_ = [("history", C.c_void_p), ("history_stride", C.c_int64), ("max_history", C.c_int32), ("history_lens", C.c_void_p), ("n_prompt", C.c_void_p),
                ("repetition", C.c_void_p), ("presence", C.c_void_p), ("frequency", C.c_void_p), ("n_bias", C.c_int32), ("bias_token", C.c_void_p),
                ("bias_value", C.c_void_p), ("allowed", C.c_void_p), ("allowed_stride", C.c_int64)]


def _load() -> C.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        path = _build.build()
    lib = C.CDLL(path)
    lib.spindlekv_status_string.restype = C.c_char_p
    lib.spindlekv_status_string.argtypes = [C.c_int32]
    lib.spindlekv_plan_layers.restype = C.c_int32
    lib.spindlekv_plan_layers.argtypes = [C.POINTER(_Config), C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.spindlekv_reserve_ratio.restype = C.c_int32
    lib.spindlekv_reserve_ratio.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.spindlekv_workspace_bytes.restype = C.c_size_t
    lib.spindlekv_workspace_bytes.argtypes = [C.POINTER(_Config), C.POINTER(_Batch), C.c_int32]
    lib.spindlekv_evict_deep.restype = C.c_int32
    lib.spindlekv_evict_deep.argtypes = [C.POINTER(_Config), C.POINTER(_Batch), _Tensor, _Tensor, C.c_void_p,
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.spindlekv_evict_deep_noalloc.restype = C.c_int32
    lib.spindlekv_evict_deep_noalloc.argtypes = [C.POINTER(_Config), C.POINTER(_Batch), _Tensor, _Tensor, C.c_void_p,
                                                 C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.spindlekv_codebook_shallow.restype = C.c_int32
    lib.spindlekv_codebook_shallow.argtypes = [C.POINTER(_Config), C.POINTER(_Batch), _Tensor, C.c_float,
                                               C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                               C.c_void_p, C.c_size_t, C.c_void_p]
    lib.spindlekv_compact.restype = C.c_int32
    lib.spindlekv_compact.argtypes = [C.POINTER(_Batch), C.c_int32, C.c_int32, _Tensor, C.c_void_p, C.c_void_p,
                                      C.c_void_p, _Tensor, C.c_void_p, C.c_void_p]
    lib.spindlekv_union_lists.restype = C.c_int32
    lib.spindlekv_union_lists.argtypes = [C.c_int32] * 7 + [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                                            C.c_void_p, C.c_void_p]
    lib.spindlekv_match_workspace_bytes.restype = C.c_size_t
    lib.spindlekv_match_workspace_bytes.argtypes = [C.POINTER(_Batch), C.c_int32]
    lib.spindlekv_codebook_match.restype = C.c_int32
    lib.spindlekv_codebook_match.argtypes = [C.POINTER(_Batch), C.c_int32, C.c_int32, _Tensor, _Tensor, C.c_void_p, C.c_int32,
                                             C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_size_t, C.c_void_p]
    lib.spindlekv_codebook_append.restype = C.c_int32
    lib.spindlekv_codebook_append.argtypes = [C.POINTER(_Batch), C.c_int32, C.c_int32, _Tensor] + [C.c_void_p] * 6 + \
                                             [_Tensor, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.spindlekv_reconstruct.restype = C.c_int32
    lib.spindlekv_reconstruct.argtypes = [C.POINTER(_Batch), C.c_int32, C.c_int32, _Tensor, C.c_void_p, C.c_void_p,
                                          _Tensor, C.c_void_p]
    lib.spindlekv_rope_table_bytes.restype = C.c_size_t
    lib.spindlekv_rope_table_bytes.argtypes = [C.c_int32, C.c_int32]
    lib.spindlekv_rope_table.restype = C.c_int32
    lib.spindlekv_rope_table.argtypes = [C.c_int32, C.c_int32, C.c_double, C.c_void_p, C.c_void_p]
    lib.spindlekv_decode_workspace_bytes.restype = C.c_size_t
    lib.spindlekv_decode_workspace_bytes.argtypes = [C.POINTER(_Batch), C.c_int32, C.c_int32, C.c_int32]
    lib.spindlekv_decode_attend.restype = C.c_int32
    lib.spindlekv_decode_attend.argtypes = [C.POINTER(_Batch), C.c_int32, C.c_int32, C.c_int32, _Tensor, C.c_void_p,
                                            _Tensor, C.c_void_p, C.c_void_p, _Tensor, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    pool, table = C.POINTER(_PagePool), C.POINTER(_PageTable)
    lib.spindlekv_pages_workspace_bytes.restype = C.c_size_t
    lib.spindlekv_pages_workspace_bytes.argtypes = [pool, table]
    lib.spindlekv_pages_resize.restype = C.c_int32
    lib.spindlekv_pages_resize.argtypes = [pool, table, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.spindlekv_pages_fork.restype = C.c_int32
    lib.spindlekv_pages_fork.argtypes = [pool, table, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.spindlekv_pages_compact.restype = C.c_int32
    lib.spindlekv_pages_compact.argtypes = [pool, table, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.spindlekv_paged_append.restype = C.c_int32
    lib.spindlekv_paged_append.argtypes = [pool, table, C.c_void_p, C.c_int32, _Tensor, _Tensor, C.c_int32, C.c_void_p, C.c_int32,
                                           C.c_int32, C.c_void_p]
    lib.spindlekv_paged_append_rotated.restype = C.c_int32
    lib.spindlekv_paged_append_rotated.argtypes = [pool, table, C.c_void_p, C.c_int32, _Tensor, _Tensor, C.c_int32, C.c_void_p, C.c_int32, C.c_int32,
                                                   C.c_void_p, C.c_int32, C.c_void_p, _Tensor, C.c_int32, _Tensor, _Tensor, C.c_void_p]
    lib.spindlekv_logits_adjust.restype = C.c_int32
    lib.spindlekv_logits_adjust.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_int64, C.POINTER(_LogitRules), C.c_void_p, C.c_int64, C.c_void_p]
    lib.spindlekv_paged_workspace_bytes.restype = C.c_size_t
    lib.spindlekv_paged_workspace_bytes.argtypes = [pool, table, C.c_int32, C.c_int32]
    lib.spindlekv_paged_attend.restype = C.c_int32
    lib.spindlekv_paged_attend.argtypes = [pool, table, C.c_int32, C.c_int32, C.c_int32, C.c_float, _Tensor, _Tensor, C.c_void_p,
                                           C.c_size_t, C.c_void_p]
    lib.spindlekv_prompt_workspace_bytes.restype = C.c_size_t
    lib.spindlekv_prompt_workspace_bytes.argtypes = [C.POINTER(_Batch), C.POINTER(_Batch)] + [C.c_int32] * 4
    lib.spindlekv_prompt_attend.restype = C.c_int32
    lib.spindlekv_prompt_attend.argtypes = [C.POINTER(_Batch), C.POINTER(_Batch), C.c_int32, C.c_int32, C.c_int32, C.c_float, _Tensor, _Tensor, _Tensor, _Tensor,
                                            C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.spindlekv_beam_workspace_bytes.restype = C.c_size_t
    lib.spindlekv_beam_workspace_bytes.argtypes = [C.c_int32] * 4
    lib.spindlekv_beam_select.restype = C.c_int32
    lib.spindlekv_beam_select.argtypes = [C.c_int32] * 4 + [C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32,
                                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.spindlekv_poll_status.restype = C.c_int32
    lib.spindlekv_poll_status.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    lib.spindlekv_set_tuning.restype = C.c_int32
    lib.spindlekv_set_tuning.argtypes = [C.c_int32, C.c_int64]
    lib.spindlekv_get_tuning.restype = C.c_int64
    lib.spindlekv_get_tuning.argtypes = [C.c_int32]
    lib.spindlekv_selftest_mbarrier_timeout.restype = C.c_int32
    lib.spindlekv_selftest_mbarrier_timeout.argtypes = [C.c_void_p, C.c_int64, C.c_void_p]
    lib.spindlekv_launch_count.restype = C.c_int64
    lib.spindlekv_launch_count.argtypes = [C.c_int32]
    lib.spindlekv_timing_enable.restype = None
    lib.spindlekv_timing_enable.argtypes = [C.c_int32]
    lib.spindlekv_timing_read.restype = C.c_int32
    lib.spindlekv_timing_read.argtypes = [C.c_int32, C.c_void_p, C.c_void_p]
    return lib


_lib = _load()
LIBRARY_PATH = _build.LIB


@dataclasses.dataclass
class Config:
    n_layers: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    window: int
    n_shallow: int
    reserve_ratio: float = -1.0
    budget_tokens: float = -1.0
    beta: float = 0.05
    theta_k: float = 0.98
    theta_v: float = 0.95
    score_norm: int = 0
    per_query_head: int = 0

    def c(self) -> _Config:
        return _Config(self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim, self.window, self.n_shallow,
                       self.reserve_ratio, self.budget_tokens, self.beta, self.theta_k, self.theta_v, self.score_norm,
                       self.per_query_head)


@dataclasses.dataclass
class Batch:
    n_layers: int
    n_seqs: int
    max_len: int
    total_len: int
    cu_seqlens: Optional[torch.Tensor] = None  # device int32 [B+1]
    layer_lens: Optional[torch.Tensor] = None  # device int32 [n_layers, B] or [n_layers, B, H] (not with cu_seqlens)

    def c(self) -> _Batch:
        ptr = self.cu_seqlens.data_ptr() if self.cu_seqlens is not None else None
        ll = self.layer_lens.data_ptr() if self.layer_lens is not None else None
        heads = self.layer_lens.shape[2] if self.layer_lens is not None and self.layer_lens.dim() == 3 else 0
        return _Batch(self.n_layers, self.n_seqs, self.max_len, self.total_len, ptr, ll, heads)


def _dtype_code(t: torch.Tensor) -> int:
    dtype = t.dtype
    if dtype == torch.bfloat16:
        return BF16
    if dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def desc_bhnd(t: torch.Tensor) -> _Tensor:
    """Descriptor of a ``[layers, B, heads, rows, d]`` tensor (any strides, ``d`` contiguous)."""
    assert t.dim() == 5 and t.stride(4) == 1
    return _Tensor(t.data_ptr(), _dtype_code(t), t.stride(0), t.stride(1), t.stride(2), t.stride(3))


def desc_thd(t: torch.Tensor) -> _Tensor:
    """Descriptor of a packed ``[layers, total_tokens, heads, d]`` tensor (used with cu_seqlens)."""
    assert t.dim() == 4 and t.stride(3) == 1
    return _Tensor(t.data_ptr(), _dtype_code(t), t.stride(0), 0, t.stride(2), t.stride(1))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if type(stream) is int:
        return stream
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


try:      # the handle alone, without a stream object around it; the number alone, without a check that CUDA is initialised
    raw_stream, current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
except AttributeError:
    current_device = torch.cuda.current_device

    def raw_stream(device_index: int) -> int:
        return torch.cuda.current_stream(device_index).cuda_stream


def _check(status: int, where: str) -> None:
    if status != OK:
        raise SpindleKVError(status, where)


def spindlekv_plan_layers(cfg: Config, seq_lens: Sequence[int]):
    """Host planner: returns ``(layer_mode[m], r_c_layer[m, B], k_ctx[m, B])`` as numpy arrays."""
    B = len(seq_lens)
    lens = np.ascontiguousarray(seq_lens, dtype=np.int32)
    mode = np.zeros(cfg.n_layers, dtype=np.int32)
    ratio = np.zeros((cfg.n_layers, B), dtype=np.float64)
    k_ctx = np.zeros((cfg.n_layers, B), dtype=np.int32)
    cc = cfg.c()
    st = _lib.spindlekv_plan_layers(C.byref(cc), B, lens.ctypes.data, mode.ctypes.data, ratio.ctypes.data,
                                    k_ctx.ctypes.data)
    _check(st, "spindlekv_plan_layers")
    return mode, ratio, k_ctx


def spindlekv_reserve_ratio(seq_len: int, kept: int, entries_k: Sequence[int], entries_v: Sequence[int]):
    """Eq. (15)'s ``(r1, r2)`` of one layer from the CodeBook sizes per head (host arithmetic in the library)."""
    ek = np.ascontiguousarray(entries_k, dtype=np.int32)
    ev = np.ascontiguousarray(entries_v, dtype=np.int32)
    r1, r2 = C.c_double(0.0), C.c_double(0.0)
    st = _lib.spindlekv_reserve_ratio(int(ek.shape[0]), seq_len, kept, ek.ctypes.data, ev.ctypes.data, C.byref(r1), C.byref(r2))
    _check(st, "spindlekv_reserve_ratio")
    return float(r1.value), float(r2.value)


def spindlekv_workspace_bytes(cfg: Config, batch: Batch, which: int) -> int:
    cc, bb = cfg.c(), batch.c()
    return int(_lib.spindlekv_workspace_bytes(C.byref(cc), C.byref(bb), which))


def spindlekv_evict_deep(cfg: Config, batch: Batch, K: _Tensor, Qwin: _Tensor, k_ctx: torch.Tensor,
                         keep_idx: torch.Tensor, keep_cnt: torch.Tensor, scores: torch.Tensor,
                         ws: torch.Tensor, stream=None) -> None:
    cc, bb = cfg.c(), batch.c()
    st = _lib.spindlekv_evict_deep(C.byref(cc), C.byref(bb), K, Qwin, _ptr(k_ctx), _ptr(keep_idx), _ptr(keep_cnt),
                                   _ptr(scores), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "spindlekv_evict_deep")


NOALLOC_SCRATCH_BYTES = 8 * 1024 * 1024


def spindlekv_evict_deep_noalloc(cfg: Config, batch: Batch, K: _Tensor, Qwin: _Tensor, k_ctx: torch.Tensor,
                                 keep_idx: torch.Tensor, keep_cnt: torch.Tensor, scores: torch.Tensor,
                                 stream=None) -> None:
    """Eviction without a workspace, for callers that may not allocate device memory (a server whose
    pool owns the GPU, code under another allocator's lock): the kernels' scratch is a fixed 8 MiB
    array inside the library.  Raises ``WORKSPACE_TOO_SMALL`` when the call would use more than that
    (never on the tensor-core path, which keeps only a status block there).  Calls share the array, so
    calls that could overlap on the GPU must be ordered by the caller; ``spindlekv_poll_status(None)``
    reads the device status word of the last call."""
    cc, bb = cfg.c(), batch.c()
    st = _lib.spindlekv_evict_deep_noalloc(C.byref(cc), C.byref(bb), K, Qwin, _ptr(k_ctx), _ptr(keep_idx),
                                           _ptr(keep_cnt), _ptr(scores), _stream(stream))
    _check(st, "spindlekv_evict_deep_noalloc")


def spindlekv_codebook_shallow(cfg: Config, batch: Batch, Gamma: _Tensor, theta: float, mag: torch.Tensor,
                               ref: torch.Tensor, centre_idx: torch.Tensor, n_entries: torch.Tensor,
                               ws: torch.Tensor, adj_bits: Optional[torch.Tensor] = None, stream=None) -> None:
    cc, bb = cfg.c(), batch.c()
    st = _lib.spindlekv_codebook_shallow(C.byref(cc), C.byref(bb), Gamma, theta, _ptr(mag), _ptr(ref),
                                         _ptr(centre_idx), _ptr(n_entries), _ptr(adj_bits), _ptr(ws),
                                         ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "spindlekv_codebook_shallow")


def spindlekv_compact(batch: Batch, n_heads: int, head_dim: int, src: _Tensor, idx: torch.Tensor,
                      cnt: torch.Tensor, dst: _Tensor, divide_by: Optional[torch.Tensor] = None,
                      dst_cu_seqlens: Optional[torch.Tensor] = None, stream=None) -> None:
    bb = batch.c()
    st = _lib.spindlekv_compact(C.byref(bb), n_heads, head_dim, src, _ptr(idx), _ptr(cnt), _ptr(divide_by), dst,
                                _ptr(dst_cu_seqlens), _stream(stream))
    _check(st, "spindlekv_compact")


def spindlekv_union_lists(n_layers: int, n_seqs: int, n_heads: int, idx_in: torch.Tensor, cnt_in: torch.Tensor,
                          seq_in: int, idx_out: torch.Tensor, cnt_out: torch.Tensor, seq_out: int, stream=None,
                          lists_inner: bool = False) -> None:
    """``idx_in [n_lists, L, H, t_in]``, ``cnt_in [n_lists, L, B, H]`` (``lists_inner``: ``[L, H, n_lists, t_in]`` and
    ``[L, B, H, n_lists]``) -> ``idx_out [L, H, t_out]``, ``cnt_out [L, B, H]``."""
    n_lists = idx_in.shape[2] if lists_inner else idx_in.shape[0]
    st = _lib.spindlekv_union_lists(n_layers, n_seqs, n_heads, n_lists, 1 if lists_inner else 0, idx_in.shape[-1], seq_in,
                                    _ptr(idx_in), _ptr(cnt_in), idx_out.shape[-1], seq_out, _ptr(idx_out), _ptr(cnt_out),
                                    _stream(stream))
    _check(st, "spindlekv_union_lists")


def spindlekv_match_workspace_bytes(batch: Batch, n_heads: int) -> int:
    bb = batch.c()
    return int(_lib.spindlekv_match_workspace_bytes(C.byref(bb), n_heads))


def spindlekv_codebook_match(batch: Batch, n_heads: int, head_dim: int, G_new: _Tensor, Cb: _Tensor, n_entries: torch.Tensor,
                             c_rows: int, theta: float, mag_new: torch.Tensor, ref_new: torch.Tensor,
                             left_idx: torch.Tensor, left_cnt: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    bb = batch.c()
    st = _lib.spindlekv_codebook_match(C.byref(bb), n_heads, head_dim, G_new, Cb, _ptr(n_entries), c_rows, theta,
                                       _ptr(mag_new), _ptr(ref_new), _ptr(left_idx), _ptr(left_cnt), _ptr(ws),
                                       ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "spindlekv_codebook_match")


def spindlekv_codebook_append(batch: Batch, n_heads: int, head_dim: int, G_left: _Tensor, mag_left: torch.Tensor,
                              ref_left: torch.Tensor, centre_left: torch.Tensor, n_left_entries: torch.Tensor,
                              left_idx: torch.Tensor, left_cnt: torch.Tensor, Cb: _Tensor, c_rows: int,
                              n_entries: torch.Tensor, ref_new: torch.Tensor, stream=None) -> None:
    bb = batch.c()
    st = _lib.spindlekv_codebook_append(C.byref(bb), n_heads, head_dim, G_left, _ptr(mag_left), _ptr(ref_left),
                                        _ptr(centre_left), _ptr(n_left_entries), _ptr(left_idx), _ptr(left_cnt), Cb,
                                        c_rows, _ptr(n_entries), _ptr(ref_new), _stream(stream))
    _check(st, "spindlekv_codebook_append")


def spindlekv_reconstruct(batch: Batch, n_heads: int, head_dim: int, Cb: _Tensor, ref: torch.Tensor,
                          mag: torch.Tensor, dst: _Tensor, stream=None) -> None:
    bb = batch.c()
    st = _lib.spindlekv_reconstruct(C.byref(bb), n_heads, head_dim, Cb, _ptr(ref), _ptr(mag), dst, _stream(stream))
    _check(st, "spindlekv_reconstruct")


def spindlekv_rope_table_bytes(head_dim: int, n_positions: int) -> int:
    return int(_lib.spindlekv_rope_table_bytes(head_dim, n_positions))


def spindlekv_rope_table(head_dim: int, n_positions: int, base: float, table: torch.Tensor, stream=None) -> None:
    """Fills ``table`` (``[n_positions, head_dim/2, 2]`` fp32: cos, sin) for ``spindlekv_decode_attend``."""
    _check(_lib.spindlekv_rope_table(head_dim, n_positions, base, _ptr(table), _stream(stream)), "spindlekv_rope_table")


def spindlekv_decode_workspace_bytes(batch: Batch, n_q_heads: int, n_kv_heads: int, head_dim: int) -> int:
    bb = batch.c()
    return int(_lib.spindlekv_decode_workspace_bytes(C.byref(bb), n_q_heads, n_kv_heads, head_dim))


def spindlekv_decode_attend(batch: Batch, n_q_heads: int, n_kv_heads: int, head_dim: int, q: _Tensor, pos_q: torch.Tensor,
                            C_K: _Tensor, ref_K: torch.Tensor, mag_K: torch.Tensor, C_V: _Tensor, ref_V: torch.Tensor,
                            mag_V: torch.Tensor, positions: Optional[torch.Tensor], rope_table: torch.Tensor,
                            out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """One decode step over the replaced cache; ``rope_table`` is ``[n_positions, head_dim/2, 2]`` fp32."""
    bb = batch.c()
    st = _lib.spindlekv_decode_attend(C.byref(bb), n_q_heads, n_kv_heads, head_dim, q, _ptr(pos_q), C_K, _ptr(ref_K),
                                      _ptr(mag_K), C_V, _ptr(ref_V), _ptr(mag_V), _ptr(positions), _ptr(rope_table),
                                      rope_table.shape[0], _ptr(out), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "spindlekv_decode_attend")


class PagePool:
    """The pages of an 8-bit cache.  ``k_codes``, ``v_codes``: ``[n_pages, H_kv, page_size, d]`` int8 or float8_e4m3fn;
    ``k_scale``, ``v_scale``: ``[n_pages, H_kv, page_size / 16]`` fp32; ``page_ref``: ``[n_pages]`` int32 (0: free).  All contiguous."""

    def __init__(self, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, page_ref: torch.Tensor):
        formats = {torch.int8: PAGED_INT8, torch.float8_e4m3fn: PAGED_E4M3}
        if k_codes.dtype not in formats or v_codes.dtype != k_codes.dtype:
            raise TypeError(f"unsupported code dtypes {k_codes.dtype}, {v_codes.dtype}")
        n, h, ps, d = k_codes.shape
        scales = (n, h, ps // PAGED_BLOCK)
        if v_codes.shape != k_codes.shape or tuple(k_scale.shape) != scales or tuple(v_scale.shape) != scales or tuple(page_ref.shape) != (n,):
            raise ValueError("the parts of a page pool do not fit together")
        if k_scale.dtype != torch.float32 or v_scale.dtype != torch.float32 or page_ref.dtype != torch.int32:
            raise TypeError("scales are fp32, reference counts int32")
        self.tensors = (k_codes, v_codes, k_scale, v_scale, page_ref)      # kept alive with the pointers
        if not all(t.is_contiguous() and t.device == k_codes.device for t in self.tensors):
            raise ValueError("the parts of a page pool are contiguous and on one device")
        self.device = k_codes.device
        self.c = _PagePool(*(t.data_ptr() for t in self.tensors), n, ps, h, d, formats[k_codes.dtype])


class PageTable:
    """``pages``: ``[n_layers, n_seqs, max_pages]`` int32, ``lens``: ``[n_layers, n_seqs]`` int32, both contiguous."""

    def __init__(self, pages: torch.Tensor, lens: torch.Tensor):
        if pages.dim() != 3 or tuple(lens.shape) != tuple(pages.shape[:2]) or pages.dtype != torch.int32 or lens.dtype != torch.int32:
            raise ValueError("pages [n_layers, n_seqs, max_pages] and lens [n_layers, n_seqs] are int32 and fit together")
        if not (pages.is_contiguous() and lens.is_contiguous() and pages.device == lens.device):
            raise ValueError("pages and lens are contiguous and on one device")
        self.pages, self.lens, self.n_layers = pages, lens, pages.shape[0]
        self.c = _PageTable(pages.data_ptr(), lens.data_ptr(), *pages.shape)


def _bytes(ws: torch.Tensor) -> int:
    return ws.nbytes


def spindlekv_pages_workspace_bytes(pool: PagePool, table: PageTable) -> int:
    return int(_lib.spindlekv_pages_workspace_bytes(pool.c, table.c))


def spindlekv_pages_resize(pool: PagePool, table: PageTable, new_lens: Optional[torch.Tensor], add: int, start: torch.Tensor,
                           ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spindlekv_pages_resize(pool.c, table.c, _ptr(new_lens), add, _ptr(start), _ptr(ws), _bytes(ws), _stream(stream)),
           "spindlekv_pages_resize")


def spindlekv_pages_fork(pool: PagePool, table: PageTable, parent: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spindlekv_pages_fork(pool.c, table.c, _ptr(parent), _ptr(ws), _bytes(ws), _stream(stream)), "spindlekv_pages_fork")


def spindlekv_pages_compact(pool: PagePool, table: PageTable, n_live: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spindlekv_pages_compact(pool.c, table.c, _ptr(n_live), _ptr(ws), _bytes(ws), _stream(stream)), "spindlekv_pages_compact")


def spindlekv_paged_append(pool: PagePool, table: PageTable, start: torch.Tensor, max_new: int, K: _Tensor, V: _Tensor, n_rows: int,
                           idx: Optional[torch.Tensor] = None, idx_seq: int = 0, stream=None) -> None:
    """``idx``: ``[n_layers, H_kv, T]`` row numbers, sequence ``s`` from column ``s * idx_seq`` on (``keep_idx`` of an eviction)."""
    _check(_lib.spindlekv_paged_append(pool.c, table.c, _ptr(start), max_new, K, V, n_rows, _ptr(idx), 0 if idx is None else idx.shape[-1],
                                       idx_seq, _stream(stream)), "spindlekv_paged_append")


NO_TENSOR = _Tensor(None, F32, 0, 0, 0, 0)


def spindlekv_paged_append_rotated(pool: PagePool, table: PageTable, start: torch.Tensor, max_new: int, K: _Tensor, V: _Tensor, n_rows: int, rope_table: torch.Tensor,
                                   first_pos: Optional[torch.Tensor] = None, K_out: _Tensor = NO_TENSOR, n_q_heads: int = 0, Q: _Tensor = NO_TENSOR,
                                   Q_out: _Tensor = NO_TENSOR, idx: Optional[torch.Tensor] = None, idx_seq: int = 0, stream=None) -> None:
    """``rope_table``: ``[n_positions, head_dim/2, 2]`` fp32; ``idx`` as for ``spindlekv_paged_append``."""
    _check(_lib.spindlekv_paged_append_rotated(pool.c, table.c, _ptr(start), max_new, K, V, n_rows, _ptr(idx), 0 if idx is None else idx.shape[-1], idx_seq,
                                               _ptr(rope_table), rope_table.shape[0], _ptr(first_pos), K_out, n_q_heads, Q, Q_out, _stream(stream)),
           "spindlekv_paged_append_rotated")


def spindlekv_paged_workspace_bytes(pool: PagePool, table: PageTable, n_q_heads: int, n_rows: int) -> int:
    return int(_lib.spindlekv_paged_workspace_bytes(pool.c, table.c, n_q_heads, n_rows))


def spindlekv_paged_attend(pool: PagePool, table: PageTable, n_q_heads: int, n_rows: int, max_len: int, scale: float, q: _Tensor,
                           out: _Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(_lib.spindlekv_paged_attend(pool.c, table.c, n_q_heads, n_rows, max_len, scale, q, out, _ptr(ws), _bytes(ws), _stream(stream)),
           "spindlekv_paged_attend")


def spindlekv_logits_adjust(logits: torch.Tensor, out: torch.Tensor, rules: _LogitRules, stream=None) -> None:
    """``logits``, ``out``: ``[n_rows, vocab]`` with any row stride, the rows contiguous."""
    _check(_lib.spindlekv_logits_adjust(logits.shape[0], logits.shape[1], _ptr(logits), _dtype_code(logits), logits.stride(0), rules, _ptr(out), out.stride(0),
                                        _stream(stream)), "spindlekv_logits_adjust")


def spindlekv_prompt_workspace_bytes(keys: Batch, rows: Optional[Batch], n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: int) -> int:
    kk, rr = keys.c(), None if rows is None else rows.c()
    return int(_lib.spindlekv_prompt_workspace_bytes(kk, rr, n_q_heads, n_kv_heads, head_dim, dtype))


def spindlekv_prompt_attend(keys: Batch, rows: Optional[Batch], n_q_heads: int, n_kv_heads: int, head_dim: int, scale: float, q: _Tensor, K: _Tensor, V: _Tensor,
                            out: _Tensor, lse: Optional[torch.Tensor], ws: torch.Tensor, stream=None) -> None:
    """``lse``: ``[n_layers, n_q_heads, T]`` fp32 or None.  ``rows`` None: every token is a row."""
    if isinstance(keys, Batch):
        keys = keys.c()
    if isinstance(rows, Batch):
        rows = rows.c()
    _check(_lib.spindlekv_prompt_attend(keys, rows, n_q_heads, n_kv_heads, head_dim, scale, q, K, V, out, _ptr(lse), _ptr(ws), _bytes(ws), _stream(stream)),
           "spindlekv_prompt_attend")


def spindlekv_beam_workspace_bytes(n_seqs: int, n_beams: int, vocab: int, n_out: int) -> int:
    return int(_lib.spindlekv_beam_workspace_bytes(n_seqs, n_beams, vocab, n_out))


def spindlekv_beam_select(n_seqs: int, n_beams: int, vocab: int, n_out: int, logits: torch.Tensor, score: torch.Tensor,
                          finished: Optional[torch.Tensor], eos: int, out_score: torch.Tensor, out_parent: torch.Tensor,
                          out_token: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """``logits``: ``[n_seqs * n_beams, vocab]`` with any row stride, the row itself contiguous."""
    _check(_lib.spindlekv_beam_select(n_seqs, n_beams, vocab, n_out, _ptr(logits), _dtype_code(logits), logits.stride(0), _ptr(score),
                                      _ptr(finished), eos, _ptr(out_score), _ptr(out_parent), _ptr(out_token), _ptr(ws), _bytes(ws),
                                      _stream(stream)), "spindlekv_beam_select")


def spindlekv_poll_status(ws: Optional[torch.Tensor]):
    """Device status word of a workspace and ``[greedy rounds, live tokens left, units done as a bit matrix, list entries built from records]``.  ``None`` reads the
    built-in scratch of ``spindlekv_evict_deep_noalloc`` on the current device."""
    status = C.c_int32(0)
    detail = (C.c_int32 * 4)()
    st = _lib.spindlekv_poll_status(_ptr(ws), C.byref(status), detail)
    _check(st, "spindlekv_poll_status")
    return int(status.value), [int(x) for x in detail]


TUNE_RECORDS_PER_TILE, TUNE_GREEDY_ROUND_CAP, TUNE_MBAR_WAIT_CYCLES, TUNE_SIM_BLOCK_PAIRS, TUNE_PAGED_WITHHOLD = range(5)


def spindlekv_set_tuning(key: int, value: int) -> None:
    """Test hook: tightens one of the library's limits (``value < 0`` restores the default)."""
    _check(_lib.spindlekv_set_tuning(key, value), "spindlekv_set_tuning")


def spindlekv_get_tuning(key: int) -> int:
    return int(_lib.spindlekv_get_tuning(key))


def spindlekv_selftest_mbarrier_timeout(ws: torch.Tensor, limit: int, stream=None) -> None:
    """Test hook: a shared-memory barrier nobody arrives on; must leave TIMEOUT in the status word of ``ws``."""
    _check(_lib.spindlekv_selftest_mbarrier_timeout(_ptr(ws), limit, _stream(stream)), "spindlekv_selftest_mbarrier_timeout")


def spindlekv_launch_count(reset: bool = False) -> int:
    return int(_lib.spindlekv_launch_count(1 if reset else 0))


def spindlekv_timing_enable(on: bool) -> None:
    _lib.spindlekv_timing_enable(1 if on else 0)


def spindlekv_timing_read():
    """``{kernel class: (milliseconds, launches)}`` since timing was enabled."""
    out = {}
    for i, name in enumerate(KERNEL_CLASSES):
        ms, n = C.c_double(0.0), C.c_int64(0)
        _check(_lib.spindlekv_timing_read(i, C.byref(ms), C.byref(n)), "spindlekv_timing_read")
        out[name] = (float(ms.value), int(n.value))
    return out


def row_words(max_len: int) -> int:
    """Words per row of the adjacency bit matrix."""
    return 4 * ((max_len + 127) // 128)
