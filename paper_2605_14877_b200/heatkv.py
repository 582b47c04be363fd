"""ctypes binding of libheatkv: argument marshalling only, same names as the C entry points.

Tensors are passed as device pointers (`tensor.data_ptr()`), streams as the raw
`cudaStream_t` of `torch.cuda.current_stream()` unless one is given.  Every function raises
`HeatKVError` when the library returns a negative status.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np
import torch

__all__ = [
    "HeatKVError", "Config", "Strides", "AllocStats", "lib_path", "exported_symbols",
    "LAYOUT_RAGGED", "LAYOUT_PAGED", "POLICY_HEATKV", "POLICY_BINARY", "POLICY_NAIVE", "POLICY_EXPLICIT",
    "ACCOUNT_PHYSICAL", "ACCOUNT_LITERAL", "KERNEL_AUTO", "KERNEL_GENERIC", "KERNEL_TCGEN05",
    "MAX_K", "MAX_BATCH", "PAGE_TOKENS",
    "heatkv_create", "heatkv_destroy", "heatkv_calibrate_scores", "heatkv_calibrate_scores_steps", "heatkv_calibrate_scores_static",
    "heatkv_finalize_scores", "heatkv_build_schedule", "heatkv_schedule_free", "heatkv_schedule_masks", "heatkv_schedule_footprint",
    "heatkv_schedule_plan", "heatkv_schedule_plan_fp8", "heatkv_seq_open", "heatkv_seq_close", "heatkv_append_compact", "heatkv_scale_attention",
    "heatkv_attention_append", "heatkv_split_plan", "heatkv_lone_plan",
    "heatkv_cache_bytes", "heatkv_retained_indices", "heatkv_export_head", "heatkv_export_head_fp8", "heatkv_allocator_stats",
    "CACHE_BF16", "CACHE_FP8_E4M3", "heatkv_launch_count", "heatkv_kernel_launches", "heatkv_pair_launches", "heatkv_lone_launches", "heatkv_last_attention", "heatkv_rank_dispersion", "heatkv_seq_reservation",
    "KernelStats", "AttentionForm", "ATTENTION_NONE", "ATTENTION_GENERIC", "ATTENTION_TCGEN05", "ATTENTION_CTA_PAIRS",
    "heatkv_selftest_wait_expiry", "heatkv_device_status", "heatkv_strerror", "heatkv_attention_split", "arena_bytes_for",
    "PagedPool", "PagedBatch", "TokenStrides", "DTYPE_BF16", "DTYPE_FP16", "PAGED_MAX_SEQ", "PAGED_MAX_SELECT", "heatkv_paged_tables",
    "heatkv_paged_release", "heatkv_paged_store", "heatkv_paged_workspace_bytes", "heatkv_paged_attention", "heatkv_paged_select",
    "heatkv_paged_sparse_attention", "heatkv_paged_status", "heatkv_paged_selftest_wait_expiry",
]

MAX_K, MAX_BATCH, PAGE_TOKENS = 16, 128, 64
CACHE_BF16, CACHE_FP8_E4M3 = 0, 1
LAYOUT_RAGGED, LAYOUT_PAGED = 0, 1
POLICY_HEATKV, POLICY_BINARY, POLICY_NAIVE, POLICY_EXPLICIT = 0, 1, 2, 3
ACCOUNT_PHYSICAL, ACCOUNT_LITERAL = 0, 1
KERNEL_AUTO, KERNEL_GENERIC, KERNEL_TCGEN05 = 0, 1, 2


class HeatKVError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {heatkv_strerror(status)} ({status})")


class Config(C.Structure):
    _fields_ = [("L", C.c_int32), ("H", C.c_int32), ("d", C.c_int32), ("K", C.c_int32),
                ("t", C.c_int32 * MAX_K), ("s", C.c_int32), ("layout", C.c_int32), ("kernel", C.c_int32),
                ("sm_scale", C.c_float), ("arena", C.c_void_p), ("arena_bytes", C.c_uint64),
                ("meta_bytes", C.c_uint64), ("scratch_bytes", C.c_uint64),
                ("cache_dtype", C.c_int32), ("reserved0", C.c_int32), ("stage_bytes", C.c_uint64)]

    @classmethod
    def make(cls, L: int, H: int, d: int, t: Sequence[int], s: int, layout: int = LAYOUT_PAGED,
             kernel: int = KERNEL_AUTO, sm_scale: float = 0.0, arena: Optional[torch.Tensor] = None,
             meta_bytes: int = 0, scratch_bytes: int = 0, cache_dtype: int = 0, stage_bytes: int = 0) -> "Config":
        cfg = cls()
        cfg.L, cfg.H, cfg.d, cfg.K, cfg.s = L, H, d, len(t), s
        for i, v in enumerate(t):
            cfg.t[i] = int(v)
        cfg.layout, cfg.kernel, cfg.sm_scale, cfg.meta_bytes = layout, kernel, sm_scale, meta_bytes
        cfg.scratch_bytes = scratch_bytes
        cfg.cache_dtype, cfg.stage_bytes = cache_dtype, stage_bytes
        if arena is not None:
            cfg.arena = arena.data_ptr()
            cfg.arena_bytes = arena.numel() * arena.element_size()
        return cfg


class Strides(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("q_seq", "q_head", "q_tok", "kv_seq", "kv_head", "kv_tok",
                                         "o_seq", "o_head", "o_tok")]

    @classmethod
    def of(cls, q: torch.Tensor, kv: torch.Tensor, o: Optional[torch.Tensor] = None) -> "Strides":
        """Strides of [n_seq, H, t, d] views (d contiguous)."""
        sq, skv = q.stride(), kv.stride()
        so = sq if o is None else o.stride()
        for s in (sq, skv, so):
            assert len(s) == 4 and s[3] == 1
        return cls(*sq[:3], *skv[:3], *so[:3])


class AllocStats(C.Structure):
    _fields_ = [("pool_rows", C.c_uint64), ("reserved_rows", C.c_uint64), ("used_tokens", C.c_uint64),
                ("peak_reserved_rows", C.c_uint64), ("meta_bytes_used", C.c_uint64),
                ("open_seqs", C.c_uint32), ("plans", C.c_uint32)]


class KernelStats(C.Structure):
    _fields_ = [("tcgen05_attention_ready", C.c_uint32), ("tcgen05_calibration_ready", C.c_uint32),
                ("attention_tcgen05", C.c_uint64), ("attention_generic", C.c_uint64),
                ("calibration_tcgen05", C.c_uint64), ("calibration_generic", C.c_uint64),
                ("append", C.c_uint64), ("compact", C.c_uint64), ("other", C.c_uint64)]


ATTENTION_NONE, ATTENTION_GENERIC, ATTENTION_TCGEN05, ATTENTION_CTA_PAIRS = 0, 1, 2, 3


class AttentionForm(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("items", C.c_int32), ("longest_piece", C.c_int32), ("lone", C.c_int32)]


# ---- paged cache of requests of any length
PAGED_MAX_SEQ, PAGED_MAX_SELECT = 4096, 32768
DTYPE_BF16, DTYPE_FP16 = 0, 1
_DTYPES = {torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_FP16}


def _expect(x: torch.Tensor, dtype: torch.dtype, shape, what: str) -> torch.Tensor:
    """x, if it has the type and shape (None: any extent); the library sees pointers only."""
    if x.dtype != dtype or x.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, x.shape)):
        raise ValueError(f"{what}: expected {dtype} {tuple(shape)}, got {x.dtype} {tuple(x.shape)}")
    return x


# Checks of the paged calls.  The calls that a model's step repeats make the same checks in C first (_paged) and come here where one fails,
# to say which (a table call 9.4 us from Python through ctypes, 6.1 from C).
_I32 = torch.int32


def _vector(x: torch.Tensor, n: int, what: str) -> int:
    """Address of a contiguous int32 vector of n entries."""
    if x.dtype is not _I32 or x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous int32 vector of {n}, got {x.dtype} {tuple(x.shape)}")
    return x.data_ptr()


def _table(x: torch.Tensor, n: int):
    """(address, row stride, columns) of a block table of n rows."""
    if x.dtype is not _I32 or x.dim() != 2 or x.size(0) != n or x.stride(1) != 1:
        raise ValueError(f"block_table: expected int32 [{n}, pages] with contiguous rows, got {x.dtype} {tuple(x.shape)}")
    pages = x.size(1)
    return x.data_ptr(), (x.stride(0) if n > 1 else pages), pages


def _packed(x: torch.Tensor, dtype: torch.dtype, shape, what: str) -> torch.Tensor:
    if not _expect(x, dtype, shape, what).is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor")
    return x


def _one_device(tensors) -> int:
    """The index of the device that all of them lie on (-1: host memory)."""
    on = {x.get_device() for x in tensors}
    if len(on) > 1:
        raise ValueError("tensors on more than one device")
    return on.pop()


class PagedPool(C.Structure):
    """One layer's pages: k, v [n_pages, n_kv_heads, 64, d] views (d contiguous, any other strides) and, for page selection,
    their summaries.  Keeps the tensors alive."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_code", C.c_void_p), ("k_scale", C.c_void_p),
                ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("row_stride", C.c_int64),
                ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32)]

    @classmethod
    def make(cls, k: torch.Tensor, v: torch.Tensor, k_code: Optional[torch.Tensor] = None,
             k_scale: Optional[torch.Tensor] = None) -> "PagedPool":
        if k.dtype not in _DTYPES:
            raise ValueError(f"k: expected bfloat16 or float16, got {k.dtype}")
        _expect(k, k.dtype, (None, None, PAGE_TOKENS, None), "k")
        _expect(v, k.dtype, k.shape, "v")
        if k.stride() != v.stride() or k.stride(3) != 1:
            raise ValueError("k, v: expected equal strides, the last dimension contiguous")
        p = cls()
        p.tensors = (k, v, k_code, k_scale)
        p.device = _one_device(x for x in p.tensors if x is not None)
        p.k, p.v = k.data_ptr(), v.data_ptr()
        if k_code is not None:
            p.k_code = _packed(k_code, torch.int8, (k.shape[0], k.shape[1], k.shape[3]), "k_code").data_ptr()
        if k_scale is not None:
            p.k_scale = _packed(k_scale, torch.float32, (k.shape[0], k.shape[1]), "k_scale").data_ptr()
        p.page_stride, p.head_stride, p.row_stride = k.stride()[:3]
        p.n_pages, p.n_kv_heads, p.d, p.dtype = k.shape[0], k.shape[1], k.shape[3], _DTYPES[k.dtype]
        p.torch_dtype, p.addr = k.dtype, C.addressof(p)
        return p


class PagedBatch(C.Structure):
    """The requests of a step: int32 tensors q_begin [n_seq + 1], kv_len [n_seq], block_table [n_seq, pages]; n_tokens rows in the token
    tensors, max_new new tokens in the longest request.  Keeps the tensors alive."""
    _fields_ = [("q_begin", C.c_void_p), ("kv_len", C.c_void_p), ("block_table", C.c_void_p), ("table_stride", C.c_int64),
                ("n_seq", C.c_int32), ("table_pages", C.c_int32), ("n_tokens", C.c_int32), ("max_new", C.c_int32)]

    @classmethod
    def make(cls, q_begin: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, n_tokens: int, max_new: int) -> "PagedBatch":
        n = kv_len.shape[0]
        _packed(q_begin, torch.int32, (n + 1,), "q_begin")
        _packed(kv_len, torch.int32, (n,), "kv_len")
        _expect(block_table, torch.int32, (n, None), "block_table")
        if block_table.stride(1) != 1:
            raise ValueError("block_table: expected contiguous rows")
        b = cls()
        b.tensors = (q_begin, kv_len, block_table)
        b.device = _one_device(b.tensors)
        b.q_begin, b.kv_len, b.block_table = q_begin.data_ptr(), kv_len.data_ptr(), block_table.data_ptr()
        b.table_stride = block_table.stride(0) if n > 1 else block_table.shape[1]
        b.n_seq, b.table_pages, b.n_tokens, b.max_new = n, block_table.shape[1], int(n_tokens), int(max_new)
        b.addr = C.addressof(b)
        return b


class TokenStrides(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("q_tok", "q_head", "o_tok", "o_head")]


def lib_path() -> str:
    return os.path.join(os.path.dirname(os.path.abspath(__file__)), "libheatkv.so")


def exported_symbols():
    """Names declared in include/heatkv.h, in declaration order."""
    return ["heatkv_create", "heatkv_destroy", "heatkv_calibrate_scores", "heatkv_calibrate_scores_steps", "heatkv_calibrate_scores_static",
            "heatkv_finalize_scores",
            "heatkv_build_schedule", "heatkv_schedule_free", "heatkv_schedule_masks",
            "heatkv_schedule_footprint", "heatkv_schedule_plan", "heatkv_schedule_plan_fp8", "heatkv_seq_open", "heatkv_seq_close", "heatkv_append_compact",
            "heatkv_scale_attention", "heatkv_attention_append", "heatkv_cache_bytes", "heatkv_seq_reservation",
            "heatkv_retained_indices", "heatkv_export_head", "heatkv_export_head_fp8",
            "heatkv_attention_split", "heatkv_split_plan", "heatkv_lone_plan", "heatkv_allocator_stats", "heatkv_launch_count",
            "heatkv_kernel_launches", "heatkv_pair_launches", "heatkv_lone_launches", "heatkv_last_attention", "heatkv_rank_dispersion", "heatkv_selftest_wait_expiry", "heatkv_device_status",
            "heatkv_strerror",
            "heatkv_paged_tables", "heatkv_paged_release", "heatkv_paged_store", "heatkv_paged_workspace_bytes", "heatkv_paged_attention",
            "heatkv_paged_select", "heatkv_paged_sparse_attention", "heatkv_paged_status", "heatkv_paged_selftest_wait_expiry"]


def _load() -> C.CDLL:
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python paper_2605_14877_b200/build.py` "
                          "(the CUDA library is the only implementation; there is no fallback)")
    return C.CDLL(path)


_lib = _load()
from . import _paged  # noqa: E402  (behind the library that it is linked to)

_lib.heatkv_strerror.restype = C.c_char_p
_lib.heatkv_strerror.argtypes = [C.c_int]
_P = C.c_void_p
_lib.heatkv_create.argtypes = [C.POINTER(Config), _P, C.POINTER(_P)]
_lib.heatkv_destroy.argtypes = [_P]
_lib.heatkv_calibrate_scores.argtypes = [_P, C.c_int, C.c_int, C.c_int, _P, _P, _P, C.POINTER(Strides), _P, _P, _P, _P]
_lib.heatkv_calibrate_scores_static.argtypes = [_P, C.c_int, C.c_int, C.c_int, _P, _P, C.POINTER(Strides), _P, _P, _P]
_lib.heatkv_calibrate_scores_steps.argtypes = [_P, C.c_int, C.c_int, C.c_int, C.c_int, _P, _P, C.POINTER(Strides), _P, _P, _P]
_lib.heatkv_finalize_scores.argtypes = [_P, _P, C.c_int, _P, _P, _P, _P]
_lib.heatkv_build_schedule.argtypes = [C.POINTER(Config), _P, _P, C.c_int, C.c_int, C.c_double, _P, C.POINTER(_P)]
_lib.heatkv_schedule_free.argtypes = [_P]
_lib.heatkv_schedule_masks.argtypes = [_P, _P, _P, _P, C.POINTER(C.c_int64)]
_lib.heatkv_schedule_footprint.argtypes = [_P, C.c_int, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
_lib.heatkv_schedule_plan.argtypes = [_P, C.c_int, _P, C.POINTER(C.c_int64)]
_lib.heatkv_schedule_plan_fp8.argtypes = [_P, _P, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
_lib.heatkv_seq_open.argtypes = [_P, _P, _P, C.POINTER(C.c_int)]
_lib.heatkv_seq_close.argtypes = [_P, C.c_int]
_lib.heatkv_append_compact.argtypes = [_P, C.POINTER(C.c_int), C.c_int, C.c_int, C.c_int, _P, _P, C.POINTER(Strides), _P]
_lib.heatkv_scale_attention.argtypes = [_P, C.POINTER(C.c_int), C.c_int, C.c_int, C.c_int, _P, _P, _P,
                                        C.POINTER(Strides), _P, _P, _P]
_lib.heatkv_attention_append.argtypes = [_P, C.POINTER(C.c_int), C.c_int, C.c_int, C.c_int, _P, _P, _P,
                                         C.POINTER(Strides), _P, _P, _P]
_lib.heatkv_split_plan.argtypes = [C.POINTER(C.c_int32), C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_uint64, C.c_uint64,
                                   C.POINTER(C.c_int32), C.POINTER(C.c_double), C.POINTER(C.c_double)]
_lib.heatkv_lone_plan.argtypes = [C.POINTER(C.c_int32), C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_uint64, C.c_uint64,
                                  C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
_lib.heatkv_attention_split.argtypes = [_P, C.POINTER(C.c_int), C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int32),
                                        C.POINTER(C.c_int32)]
_lib.heatkv_cache_bytes.argtypes = [_P, C.c_int, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
_lib.heatkv_retained_indices.argtypes = [_P, C.c_int, C.c_int, C.c_int, _P, C.POINTER(C.c_int)]
_lib.heatkv_export_head.argtypes = [_P, C.c_int, C.c_int, C.c_int, _P, _P, _P]
_lib.heatkv_export_head_fp8.argtypes = [_P, C.c_int, C.c_int, C.c_int, _P, _P, _P, _P, _P]
_lib.heatkv_allocator_stats.argtypes = [_P, C.POINTER(AllocStats)]
_lib.heatkv_launch_count.argtypes = [_P, C.POINTER(C.c_uint64)]
_lib.heatkv_pair_launches.argtypes = [_P, C.POINTER(C.c_uint64)]
_lib.heatkv_lone_launches.argtypes = [_P, C.POINTER(C.c_uint64)]
_lib.heatkv_last_attention.argtypes = [_P, C.POINTER(AttentionForm)]
_lib.heatkv_device_status.argtypes = [_P, _P]
_lib.heatkv_selftest_wait_expiry.argtypes = [_P, _P]
_lib.heatkv_kernel_launches.argtypes = [_P, C.POINTER(KernelStats)]
_lib.heatkv_rank_dispersion.argtypes = [_P, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, _P]
_lib.heatkv_seq_reservation.argtypes = [_P, C.c_int, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
_I, _L = C.c_int, C.c_int64
_lib.heatkv_paged_tables.argtypes = [_P, _P, _I, _P, _I, _P, _P, _P, _L, _I, _P, _P, _P, _P, _I, _P]
_lib.heatkv_paged_release.argtypes = [_P, _P, _I, _P, _L, _I, _P, _I, _P, _P, _P]
_lib.heatkv_paged_store.argtypes = [_P, _P, _P, _L, _L, _P, _I, _P]
_lib.heatkv_paged_workspace_bytes.argtypes = [_P, _P, _I, C.POINTER(C.c_uint64)]
_lib.heatkv_paged_attention.argtypes = [_P, _P, _I, _P, _P, _I, C.c_float, _P, _P, _P, C.c_uint64, _P]
_lib.heatkv_paged_select.argtypes = [_P, _P, _I, _P, _P, _I, _I, _I, _P, _P]
_lib.heatkv_paged_sparse_attention.argtypes = [_P, _P, _I, _P, _P, _P, _I, C.c_float, _P, _P, _P, C.c_uint64, _P]
_lib.heatkv_paged_status.argtypes = [_P, _P]
_lib.heatkv_paged_selftest_wait_expiry.argtypes = [_P, _P]
for _n in exported_symbols():
    if _n != "heatkv_strerror":
        getattr(_lib, _n).restype = C.c_int


def _stream(stream) -> int:
    if stream is None:
        # the handle itself: building the Stream object around it (torch.cuda.current_stream) costs 3 us a call
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return int(x)


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise HeatKVError(rc, where)


_paged.set_hooks(torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, torch.int32, torch.float32)


def _ids(seq_ids: Sequence[int]):
    return (C.c_int * len(seq_ids))(*[int(i) for i in seq_ids]), len(seq_ids)


def heatkv_strerror(status: int) -> str:
    return _lib.heatkv_strerror(int(status)).decode()


def arena_bytes_for(pool_rows: int, d: int, meta_bytes: int = 1 << 24, scratch_bytes: int = 1 << 26,
                    cache_dtype: int = 0, stage_bytes: int = 0) -> int:
    """Arena size that yields at least `pool_rows` rows in each of the K and V pools when the context is
    created with the same (non-zero) `meta_bytes`, `scratch_bytes` and, for the fp8 cache, `stage_bytes`."""
    rows = (pool_rows + PAGE_TOKENS - 1) // PAGE_TOKENS * PAGE_TOKENS
    fixed = (meta_bytes + 1023) // 1024 * 1024 + (scratch_bytes + 1023) // 1024 * 1024
    if cache_dtype == CACHE_FP8_E4M3:
        return fixed + stage_bytes + 2 * rows * (d + 1)
    return fixed + 2 * rows * d * 2


def heatkv_create(cfg: Config, stream=None) -> int:
    out = _P()
    _check(_lib.heatkv_create(C.byref(cfg), _stream(stream), C.byref(out)), "heatkv_create")
    return out.value


def heatkv_destroy(ctx: int) -> None:
    _check(_lib.heatkv_destroy(ctx), "heatkv_destroy")


def heatkv_calibrate_scores(ctx, layer, step, n_seq, q, k_full, v_full, strides, seg_bias, beta_accum, out,
                            stream=None) -> None:
    st = C.byref(strides) if strides is not None else None
    _check(_lib.heatkv_calibrate_scores(ctx, layer, step, n_seq, _ptr(q), _ptr(k_full), _ptr(v_full), st,
                                        _ptr(seg_bias), _ptr(beta_accum), _ptr(out), _stream(stream)),
           "heatkv_calibrate_scores")


def heatkv_calibrate_scores_steps(ctx, layer, step_begin, step_end, n_seq, q_all, k_all, strides, seg_bias, beta_accum,
                                  stream=None) -> None:
    """Eq. 2 for steps step_begin .. step_end - 1 of one layer in one call (q_all, k_all: [n_seq, H, tokens, d] with
    all scales on the token axis; seg_bias: [step_end, H, K] or None)."""
    st = C.byref(strides) if strides is not None else None
    _check(_lib.heatkv_calibrate_scores_steps(ctx, layer, step_begin, step_end, n_seq, _ptr(q_all), _ptr(k_all), st,
                                              _ptr(seg_bias), _ptr(beta_accum), _stream(stream)),
           "heatkv_calibrate_scores_steps")


def heatkv_calibrate_scores_static(ctx, layer, step, n_seq, q, k_full, strides, seg_bias, beta_accum,
                                   stream=None) -> None:
    """Same beta update as heatkv_calibrate_scores, for callers that must not allocate device memory:
    the scratch is an array inside the library.  Raises HeatKVError(-10) when the call is too large."""
    st = C.byref(strides) if strides is not None else None
    _check(_lib.heatkv_calibrate_scores_static(ctx, layer, step, n_seq, _ptr(q), _ptr(k_full), st, _ptr(seg_bias),
                                               _ptr(beta_accum), _stream(stream)), "heatkv_calibrate_scores_static")


def heatkv_finalize_scores(ctx, beta_accum, n_samples, L, H, K, stream=None):
    """Returns (beta [L,H,K,K], scas [L,H,K], cas [L,H]) as float64 numpy arrays."""
    beta = np.zeros((L, H, K, K), dtype=np.float64)
    scas = np.zeros((L, H, K), dtype=np.float64)
    cas = np.zeros((L, H), dtype=np.float64)
    _check(_lib.heatkv_finalize_scores(ctx, _ptr(beta_accum), n_samples, _ptr(beta), _ptr(scas), _ptr(cas),
                                       _stream(stream)), "heatkv_finalize_scores")
    return beta, scas, cas


def heatkv_build_schedule(cfg: Config, scas=None, cas=None, policy: int = POLICY_HEATKV,
                          accounting: int = ACCOUNT_PHYSICAL, b: float = 1.0, fraction=None) -> int:
    keep = [None if a is None else np.ascontiguousarray(a, dtype=np.float64) for a in (scas, cas, fraction)]
    out = _P()
    _check(_lib.heatkv_build_schedule(C.byref(cfg), _ptr(keep[0]), _ptr(keep[1]), policy, accounting, float(b),
                                      _ptr(keep[2]), C.byref(out)), "heatkv_build_schedule")
    return out.value


def heatkv_schedule_free(sch: int) -> None:
    _check(_lib.heatkv_schedule_free(sch), "heatkv_schedule_free")


def heatkv_schedule_masks(sch: int, K: int, L: int, H: int):
    """Returns (attn_mask [K,L,H] uint16, keep_mask [K,L,H] uint16, n_k [K] int32, budget_tokens)."""
    am = np.zeros((K, L, H), dtype=np.uint16)
    km = np.zeros((K, L, H), dtype=np.uint16)
    nk = np.zeros(K, dtype=np.int32)
    b = C.c_int64()
    _check(_lib.heatkv_schedule_masks(sch, _ptr(am), _ptr(km), _ptr(nk), C.byref(b)), "heatkv_schedule_masks")
    return am, km, nk, b.value


def heatkv_schedule_footprint(sch: int, layout: int):
    peak, rows = C.c_int64(), C.c_int64()
    _check(_lib.heatkv_schedule_footprint(sch, layout, C.byref(peak), C.byref(rows)), "heatkv_schedule_footprint")
    return peak.value, rows.value


def heatkv_schedule_plan(sch: int, layout: int) -> np.ndarray:
    """The plan tables as one int32 array (see include/heatkv.h for the layout)."""
    n = C.c_int64(0)
    _check(_lib.heatkv_schedule_plan(sch, layout, None, C.byref(n)), "heatkv_schedule_plan")
    words = np.zeros(n.value, dtype=np.int32)
    _check(_lib.heatkv_schedule_plan(sch, layout, _ptr(words), C.byref(n)), "heatkv_schedule_plan")
    return words


def heatkv_schedule_plan_fp8(sch: int):
    """(plan tables of a context with the fp8 cache as one int32 array, staging rows a sequence needs per call)."""
    n, rows = C.c_int64(0), C.c_int64(0)
    _check(_lib.heatkv_schedule_plan_fp8(sch, None, C.byref(n), None), "heatkv_schedule_plan_fp8")
    words = np.zeros(n.value, dtype=np.int32)
    _check(_lib.heatkv_schedule_plan_fp8(sch, _ptr(words), C.byref(n), C.byref(rows)), "heatkv_schedule_plan_fp8")
    return words, rows.value


def heatkv_seq_open(ctx: int, sch: int, stream=None) -> int:
    out = C.c_int()
    _check(_lib.heatkv_seq_open(ctx, sch, _stream(stream), C.byref(out)), "heatkv_seq_open")
    return out.value


def heatkv_seq_close(ctx: int, seq_id: int) -> None:
    _check(_lib.heatkv_seq_close(ctx, seq_id), "heatkv_seq_close")


def heatkv_append_compact(ctx, seq_ids, layer, step, k_new, v_new, strides=None, stream=None) -> None:
    ids, n = _ids(seq_ids)
    st = C.byref(strides) if strides is not None else None
    _check(_lib.heatkv_append_compact(ctx, ids, n, layer, step, _ptr(k_new), _ptr(v_new), st, _stream(stream)),
           "heatkv_append_compact")


def heatkv_scale_attention(ctx, seq_ids, layer, step, q, k_new, v_new, strides, seg_bias, out, stream=None) -> None:
    ids, n = _ids(seq_ids)
    st = C.byref(strides) if strides is not None else None
    _check(_lib.heatkv_scale_attention(ctx, ids, n, layer, step, _ptr(q), _ptr(k_new), _ptr(v_new), st,
                                       _ptr(seg_bias), _ptr(out), _stream(stream)), "heatkv_scale_attention")


def heatkv_attention_append(ctx, seq_ids, layer, step, q, k_new, v_new, strides, seg_bias, out, stream=None) -> None:
    """Attention of the layer at the step followed by its cache update, one launch in the paged layout."""
    ids, n = _ids(seq_ids)
    st = C.byref(strides) if strides is not None else None
    _check(_lib.heatkv_attention_append(ctx, ids, n, layer, step, _ptr(q), _ptr(k_new), _ptr(v_new), st,
                                        _ptr(seg_bias), _ptr(out), _stream(stream)), "heatkv_attention_append")


def heatkv_attention_split(ctx, seq_ids, layer, step):
    """(longest piece in 128-key tiles among the heads that are cut, 0 = whole heads; work items of the launch)
    for this attention call."""
    ids, n = _ids(seq_ids)
    a, b = C.c_int32(), C.c_int32()
    _check(_lib.heatkv_attention_split(ctx, ids, n, layer, step, C.byref(a), C.byref(b)), "heatkv_attention_split")
    return a.value, b.value


def heatkv_split_plan(tiles, n_qp: int, n_seq: int, n_sm: int = 148, per_head: bool = True,
                      max_slots: int = 1 << 40, max_ctrs: int = 1 << 40):
    """Pieces per head (tiles in descending order) and the estimated makespans (whole heads, chosen cut)."""
    n = len(tiles)
    t = (C.c_int32 * n)(*[int(x) for x in tiles])
    out = (C.c_int32 * n)()
    a, b = C.c_double(), C.c_double()
    _check(_lib.heatkv_split_plan(t, n, n_qp, n_seq, n_sm, int(per_head), max_slots, max_ctrs, out, C.byref(a), C.byref(b)),
           "heatkv_split_plan")
    return [int(x) for x in out], a.value, b.value


def heatkv_lone_plan(tiles, t_q: int, n_seq: int, n_sm: int = 148, d: int = 128, per_head: bool = True,
                     max_slots: int = 1 << 40, max_ctrs: int = 1 << 40):
    """(pieces per head, heads whose query tiles go one by one, does the launch take query tiles by themselves instead of cuts)."""
    n = len(tiles)
    t = (C.c_int32 * n)(*[int(x) for x in tiles])
    pieces, singles, lone = (C.c_int32 * n)(), (C.c_int32 * n)(), C.c_int32()
    _check(_lib.heatkv_lone_plan(t, n, t_q, n_seq, n_sm, d, int(per_head), max_slots, max_ctrs, pieces, singles, C.byref(lone)),
           "heatkv_lone_plan")
    return [int(x) for x in pieces], [bool(x) for x in singles], bool(lone.value)


def heatkv_cache_bytes(ctx: int, seq_id: int):
    """(bytes of the rows the plan placed for what the sequence stores, closed form from the schedule's masks)."""
    a, r = C.c_uint64(), C.c_uint64()
    _check(_lib.heatkv_cache_bytes(ctx, seq_id, C.byref(a), C.byref(r)), "heatkv_cache_bytes")
    return a.value, r.value


def heatkv_seq_reservation(ctx: int, seq_id: int):
    """(first pool row, rows) reserved for the sequence."""
    a, r = C.c_uint64(), C.c_uint64()
    _check(_lib.heatkv_seq_reservation(ctx, seq_id, C.byref(a), C.byref(r)), "heatkv_seq_reservation")
    return a.value, r.value


def heatkv_retained_indices(ctx: int, seq_id: int, layer: int, head: int, max_tokens: int) -> np.ndarray:
    idx = np.zeros(max_tokens, dtype=np.int32)
    n = C.c_int()
    _check(_lib.heatkv_retained_indices(ctx, seq_id, layer, head, _ptr(idx), C.byref(n)), "heatkv_retained_indices")
    return idx[: n.value].copy()


def heatkv_export_head_fp8(ctx, seq_id, layer, head, k_codes, v_codes, k_exps, v_exps, stream=None) -> None:
    _check(_lib.heatkv_export_head_fp8(ctx, seq_id, layer, head, _ptr(k_codes), _ptr(v_codes), _ptr(k_exps), _ptr(v_exps),
                                       _stream(stream)), "heatkv_export_head_fp8")


def heatkv_export_head(ctx, seq_id, layer, head, k_out, v_out, stream=None) -> None:
    _check(_lib.heatkv_export_head(ctx, seq_id, layer, head, _ptr(k_out), _ptr(v_out), _stream(stream)),
           "heatkv_export_head")


def heatkv_allocator_stats(ctx: int) -> AllocStats:
    st = AllocStats()
    _check(_lib.heatkv_allocator_stats(ctx, C.byref(st)), "heatkv_allocator_stats")
    return st


def heatkv_launch_count(ctx: int) -> int:
    n = C.c_uint64()
    _check(_lib.heatkv_launch_count(ctx, C.byref(n)), "heatkv_launch_count")
    return n.value


def heatkv_kernel_launches(ctx: int) -> KernelStats:
    st = KernelStats()
    _check(_lib.heatkv_kernel_launches(ctx, C.byref(st)), "heatkv_kernel_launches")
    return st


def heatkv_pair_launches(ctx: int) -> int:
    n = C.c_uint64()
    _check(_lib.heatkv_pair_launches(ctx, C.byref(n)), "heatkv_pair_launches")
    return n.value


def heatkv_lone_launches(ctx: int) -> int:
    n = C.c_uint64()
    _check(_lib.heatkv_lone_launches(ctx, C.byref(n)), "heatkv_lone_launches")
    return n.value


def heatkv_last_attention(ctx: int) -> AttentionForm:
    """The form in which the context's last attention call was launched."""
    f = AttentionForm()
    _check(_lib.heatkv_last_attention(ctx, C.byref(f)), "heatkv_last_attention")
    return f


def heatkv_rank_dispersion(scas_runs, s: int) -> np.ndarray:
    """scas_runs [R, L, H, K] float64 -> [K] mean standard deviation of the heads' rank positions."""
    a = np.ascontiguousarray(scas_runs, dtype=np.float64)
    R, L, H, K = a.shape
    out = np.zeros(K, dtype=np.float64)
    _check(_lib.heatkv_rank_dispersion(_ptr(a), R, L, H, K, int(s), _ptr(out)), "heatkv_rank_dispersion")
    return out


def heatkv_selftest_wait_expiry(ctx: int, stream=None) -> int:
    """Status of the bounded-wait self-test: -7 (a wait ran out, as it must) is the expected answer."""
    return _lib.heatkv_selftest_wait_expiry(ctx, _stream(stream))


def heatkv_device_status(ctx: int, stream=None) -> int:
    return _lib.heatkv_device_status(ctx, _stream(stream))


# ---------------------------------------------------------------------------------------------- paged cache
def heatkv_paged_tables(new_tokens, past_tokens, free_pages, state, state_out, block_table, q_begin, kv_len, slot_map,
                        positions=None, stream=None) -> None:
    """Pages, slots and positions of a step's new tokens, from the requests' lengths (int32 tensors on the device)."""
    rc = _paged.tables(new_tokens, past_tokens, free_pages, state, state_out, block_table, q_begin, kv_len, slot_map, positions, stream)
    if rc is not None:
        return _check(rc, "heatkv_paged_tables")
    n, n_pages, n_tokens = new_tokens.numel(), free_pages.numel(), slot_map.numel()
    table, stride, pages = _table(block_table, n)
    rc = _lib.heatkv_paged_tables(_vector(new_tokens, n, "new_tokens"), _vector(past_tokens, n, "past_tokens"), n,
                                  _vector(free_pages, n_pages, "free_pages"), n_pages, _vector(state, 4, "state"),
                                  _vector(state_out, 4, "state_out"), table, stride, pages, _vector(q_begin, n + 1, "q_begin"),
                                  _vector(kv_len, n, "kv_len"), _vector(slot_map, n_tokens, "slot_map"),
                                  None if positions is None else _vector(positions, n_tokens, "positions"), n_tokens,
                                  _on_device(stream, new_tokens, past_tokens, free_pages, state, state_out, block_table, q_begin, kv_len, slot_map,
                                             positions))
    _check(rc, "heatkv_paged_tables")


def heatkv_paged_release(kv_len, keep_len, block_table, free_pages, state, state_out, stream=None) -> None:
    """Gives back the pages that hold only tokens from keep_len on."""
    n, n_pages = kv_len.numel(), free_pages.numel()
    table, stride, pages = _table(block_table, n)
    _check(_lib.heatkv_paged_release(_vector(kv_len, n, "kv_len"), _vector(keep_len, n, "keep_len"), n, table, stride, pages,
                                     _vector(free_pages, n_pages, "free_pages"), n_pages, _vector(state, 4, "state"),
                                     _vector(state_out, 4, "state_out"),
                                     _on_device(stream, kv_len, keep_len, block_table, free_pages, state, state_out)), "heatkv_paged_release")


def heatkv_paged_store(pool: PagedPool, k_new, v_new, slot_map, stream=None) -> None:
    """K and V rows [n_tokens, n_kv_heads, d] (equal strides, d contiguous) to their slots, and the summaries of pages that fill up."""
    rc = _paged.store(pool, k_new, v_new, slot_map, stream)
    if rc is not None:
        return _check(rc, "heatkv_paged_store")
    n = slot_map.numel()
    slots = _vector(slot_map, n, "slot_map")
    _rows(k_new, pool, n, pool.n_kv_heads, "k_new")
    _rows(v_new, pool, n, pool.n_kv_heads, "v_new")
    strides = k_new.stride()
    if v_new.stride() != strides or strides[2] != 1:
        raise ValueError("k_new, v_new: expected equal strides, the last dimension contiguous")
    rc = _lib.heatkv_paged_store(pool.addr, k_new.data_ptr(), v_new.data_ptr(), strides[0], strides[1], slots, n,
                                 _on_device(stream, pool, k_new, v_new, slot_map))
    _check(rc, "heatkv_paged_store")


def heatkv_paged_workspace_bytes(pool: PagedPool, batch: PagedBatch, n_heads: int) -> int:
    """Bytes of workspace that attention over this batch needs (a zeroed uint8 tensor; it may be used again and again)."""
    out = C.c_uint64()
    _check(_lib.heatkv_paged_workspace_bytes(pool.addr, batch.addr, n_heads, C.byref(out)), "heatkv_paged_workspace_bytes")
    return out.value


def _on_device(stream, *where) -> int:
    """The stream's handle, after a look at where a call's tensors lie (tensors, pools and batches; None counts for nothing): an address
    of the host or of another GPU would fault in the kernel."""
    here = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2
    for x in where:
        if x is not None and (x.get_device() if isinstance(x, torch.Tensor) else x.device) != here:
            raise ValueError("a tensor that is not on the current CUDA device")
    return _stream(stream)


def _workspace(x) -> int:
    if not x.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    return x.data_ptr()


def _rows(x, pool, tokens, heads, what):
    """Checks [tokens, heads, d] activations (heads None: any number)."""
    if x.dtype is not pool.torch_dtype or x.dim() != 3 or x.size(0) != tokens or x.size(2) != pool.d or (heads is not None and x.size(1) != heads):
        raise ValueError(f"{what}: expected {pool.torch_dtype} [{tokens}, {'heads' if heads is None else heads}, {pool.d}], got {x.dtype} {tuple(x.shape)}")


def _token_strides(pool, batch, q, out):
    """Strides of q and out, None where both are packed."""
    tokens = batch.n_tokens
    _rows(q, pool, tokens, None, "q")
    if out is not None:
        _rows(out, pool, tokens, q.size(1), "out")
    if q.is_contiguous() and (out is None or out.is_contiguous()):
        return None
    sq, so = q.stride(), (q if out is None else out).stride()
    if sq[2] != 1 or so[2] != 1:
        raise ValueError("q, out: expected the last dimension contiguous")
    return C.byref(TokenStrides(sq[0], sq[1], so[0], so[1]))


def _lse(lse, q):
    if lse is None:
        return None
    if lse.dtype is not torch.float32 or lse.dim() != 2 or lse.size(0) != q.size(0) or lse.size(1) != q.size(1) or not lse.is_contiguous():
        raise ValueError(f"lse: expected contiguous float32 [{q.size(0)}, {q.size(1)}], got {lse.dtype} {tuple(lse.shape)}")
    return lse.data_ptr()


def _lists(sel, pool, batch):
    if sel.dtype is not _I32 or sel.dim() != 3 or sel.size(0) != batch.n_tokens or sel.size(1) != pool.n_kv_heads or not sel.is_contiguous():
        raise ValueError(f"sel: expected contiguous int32 [{batch.n_tokens}, {pool.n_kv_heads}, n_select], got {sel.dtype} {tuple(sel.shape)}")
    return sel.data_ptr(), sel.size(2)


def heatkv_paged_attention(pool: PagedPool, batch: PagedBatch, q, out, lse, workspace, causal: bool = True, sm_scale: float = 0.0,
                           stream=None) -> None:
    """out [n_tokens, n_heads, d] and (unless None) lse [n_tokens, n_heads] of the new tokens' attention over their requests' pages."""
    rc = _paged.attention(pool, batch, q, out, lse, workspace, causal, sm_scale, stream)
    if rc is not None:
        return _check(rc, "heatkv_paged_attention")
    st = _token_strides(pool, batch, q, out)
    rc = _lib.heatkv_paged_attention(pool.addr, batch.addr, q.size(1), q.data_ptr(), st, causal, sm_scale, out.data_ptr(), _lse(lse, q),
                                     _workspace(workspace), workspace.nbytes, _on_device(stream, pool, batch, q, out, lse, workspace))
    _check(rc, "heatkv_paged_attention")


def heatkv_paged_select(pool: PagedPool, batch: PagedBatch, q, sel, sink: int, local: int, stream=None) -> None:
    """sel [n_tokens, n_kv_heads, n_select]: the pages each new token attends to (places in its request's table row, ascending, -1
    after the last)."""
    rc = _paged.select(pool, batch, q, sel, sink, local, stream)
    if rc is not None:
        return _check(rc, "heatkv_paged_select")
    st = _token_strides(pool, batch, q, None)
    lists, n_select = _lists(sel, pool, batch)
    rc = _lib.heatkv_paged_select(pool.addr, batch.addr, q.size(1), q.data_ptr(), st, sink, local, n_select, lists,
                                  _on_device(stream, pool, batch, q, sel))
    _check(rc, "heatkv_paged_select")


def heatkv_paged_sparse_attention(pool: PagedPool, batch: PagedBatch, q, sel, out, lse, workspace, sm_scale: float = 0.0,
                                  stream=None) -> None:
    """heatkv_paged_attention (causal) over the pages that sel lists for each token."""
    rc = _paged.sparse_attention(pool, batch, q, sel, out, lse, workspace, sm_scale, stream)
    if rc is not None:
        return _check(rc, "heatkv_paged_sparse_attention")
    st = _token_strides(pool, batch, q, out)
    lists, n_select = _lists(sel, pool, batch)
    rc = _lib.heatkv_paged_sparse_attention(pool.addr, batch.addr, q.size(1), q.data_ptr(), st, lists, n_select, sm_scale, out.data_ptr(),
                                            _lse(lse, q), _workspace(workspace), workspace.nbytes, _on_device(stream, pool, batch, q, sel, out, lse, workspace))
    _check(rc, "heatkv_paged_sparse_attention")


def heatkv_paged_status(workspace, stream=None) -> int:
    """0, or -7 if a bounded wait of a kernel that used this workspace ran out (synchronises the stream): results since the last look are then
    not to be used, and the workspace is to be zeroed."""
    return _lib.heatkv_paged_status(workspace.data_ptr(), _on_device(stream, workspace))


def heatkv_paged_selftest_wait_expiry(workspace, stream=None) -> int:
    """-7 when the paged kernels' bounded waits, tried on a barrier that nothing signals, give up as they should; leaves the status set."""
    if workspace.nbytes < 256:
        raise ValueError("workspace: expected at least 256 bytes")
    return _lib.heatkv_paged_selftest_wait_expiry(_workspace(workspace), _on_device(stream, workspace))
