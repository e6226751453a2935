"""Python binding of libstream (argument marshalling only; every step runs in the CUDA library).

The ``stream_*`` functions mirror the C ABI in ``include/stream.h`` one to one and take torch
CUDA tensors (or raw integer addresses) where the C side takes device pointers. ``build_mask``,
``sparse_attention`` and ``run_host`` are conveniences that allocate outputs with torch and fill
in the problem struct from tensor shapes and strides. PyTorch is used for device memory and
streams only.

Masks and the sparse attention on them: ``build_mask`` ... ``mask_difference``. Dense attention and the
key-value cache of chains that are being generated: ``prompt_attention``, ``decode_attention``,
``PagedCache``, ``PagedCache8`` (8 bits an element) and the ``cache_*`` functions.
"""
from __future__ import annotations

import array
import ctypes
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libstream.so")

STREAM_OK, STREAM_ERR_INVALID_ARG, STREAM_ERR_UNSUPPORTED, STREAM_ERR_WORKSPACE, STREAM_ERR_CUDA, STREAM_ERR_DEVICE_CHECK = range(6)
STREAM_F32, STREAM_BF16 = 0, 1
IMPL = {"auto": 0, "generic": 1, "tensor": 2}
_STATUS_NAMES = ["OK", "INVALID_ARG", "UNSUPPORTED", "WORKSPACE", "CUDA", "DEVICE_CHECK"]


class StreamProblem(ctypes.Structure):
    """``stream_problem`` of stream.h."""

    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("T", ctypes.c_int64),
        ("d", ctypes.c_int32), ("block_q", ctypes.c_int32), ("block_k", ctypes.c_int32), ("k_top", ctypes.c_int32),
        ("causal", ctypes.c_int32), ("dtype", ctypes.c_int32), ("impl", ctypes.c_int32),
        ("q_stride_b", ctypes.c_int64), ("q_stride_h", ctypes.c_int64), ("q_stride_t", ctypes.c_int64),
        ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64), ("kv_stride_t", ctypes.c_int64),
    ]


_PROBLEM = struct.Struct("@iiiqiiiiiiiqqqqqq")  # StreamProblem's fields with the C compiler's padding
assert _PROBLEM.size == ctypes.sizeof(StreamProblem)


class StreamPrompt(ctypes.Structure):
    """``stream_prompt`` of stream.h."""

    _fields_ = [("n_seqs", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("d", ctypes.c_int32),
                ("total_q", ctypes.c_int64), ("total_k", ctypes.c_int64), ("causal", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("q_stride_t", ctypes.c_int64), ("q_stride_h", ctypes.c_int64), ("kv_stride_t", ctypes.c_int64),
                ("kv_stride_h", ctypes.c_int64)]


class StreamCache(ctypes.Structure):
    """``stream_cache`` of stream.h."""

    _fields_ = [("n_slots", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("d", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("stride_l", ctypes.c_int64), ("stride_p", ctypes.c_int64), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class StreamCache8(ctypes.Structure):
    """``stream_cache8`` of stream.h."""

    _fields_ = [("cache", StreamCache), ("block", ctypes.c_int32), ("reserved", ctypes.c_int32), ("scale_stride_l", ctypes.c_int64),
                ("scale_stride_p", ctypes.c_int64), ("scale_stride_b", ctypes.c_int64), ("scale_stride_h", ctypes.c_int64)]


class StreamStats(ctypes.Structure):
    """``stream_stats`` of stream.h."""

    _fields_ = [("tiles_scored", ctypes.c_uint64), ("rows", ctypes.c_uint64), ("error", ctypes.c_uint32),
                ("error_info", ctypes.c_uint32), ("tile_products", ctypes.c_uint64),
                ("tiles_fetched", ctypes.c_uint64)]


class StreamUnitRates(ctypes.Structure):
    """``stream_unit_rates`` of stream.h."""

    _fields_ = [("tma_bytes_per_clk", ctypes.c_double), ("mma_cycles_m128n64", ctypes.c_double),
                ("error", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class StreamError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"libstream: STREAM_ERR_{_STATUS_NAMES[status]}: {text}")
        self.status = status


_lib = None


def library_path() -> str:
    return _LIB_PATH


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2510_19875_b200.build` "
            "(there is no fallback path without the CUDA library)")
    lib = ctypes.CDLL(_LIB_PATH)
    P, vp, sz = ctypes.POINTER(StreamProblem), ctypes.c_void_p, ctypes.c_size_t
    lib.stream_version.restype = ctypes.c_int
    lib.stream_version.argtypes = []
    lib.stream_last_error.restype = ctypes.c_char_p
    lib.stream_last_error.argtypes = []
    lib.stream_workspace_bytes.restype = sz
    lib.stream_workspace_bytes.argtypes = [P]
    lib.stream_build_mask.restype = ctypes.c_int
    lib.stream_build_mask.argtypes = [P, vp, vp, vp, vp, vp, sz, vp]
    lib.stream_build_mask_var.restype = ctypes.c_int
    lib.stream_build_mask_var.argtypes = [P, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.stream_workspace_bytes_multi.restype = sz
    lib.stream_workspace_bytes_multi.argtypes = [P, ctypes.c_int32]
    lib.stream_build_mask_multi.restype = ctypes.c_int
    lib.stream_build_mask_multi.argtypes = [P, vp, vp, ctypes.c_int32, vp, vp, vp, vp, sz, vp]
    lib.stream_k_schedule.restype = ctypes.c_int
    lib.stream_k_schedule.argtypes = [P, ctypes.c_double, vp]
    lib.stream_effective_k.restype = ctypes.c_int
    lib.stream_effective_k.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_double, ctypes.POINTER(ctypes.c_int32)]
    lib.stream_selftest_bounded_wait.restype = ctypes.c_int
    lib.stream_selftest_bounded_wait.argtypes = [ctypes.c_int64, vp, sz, vp]
    lib.stream_probe_scratch_bytes.restype = sz
    lib.stream_probe_scratch_bytes.argtypes = []
    lib.stream_probe_unit_rates.restype = ctypes.c_int
    lib.stream_probe_unit_rates.argtypes = [vp, sz, ctypes.POINTER(StreamUnitRates), vp]
    lib.stream_build_mask_static.restype = ctypes.c_int
    lib.stream_build_mask_static.argtypes = [P, vp, vp, vp, vp, vp]
    lib.stream_sparse_attention.restype = ctypes.c_int
    lib.stream_sparse_attention.argtypes = [P, vp, vp, vp, vp, ctypes.c_float, vp, vp]
    lib.stream_read_stats.restype = ctypes.c_int
    lib.stream_read_stats.argtypes = [vp, ctypes.POINTER(StreamStats), vp]
    lib.stream_vertical_scores.restype = ctypes.c_int
    lib.stream_vertical_scores.argtypes = [P, vp, vp, vp, vp, vp, sz, vp]
    lib.stream_mask_difference.restype = ctypes.c_int
    lib.stream_mask_difference.argtypes = [ctypes.c_int64, ctypes.c_int32, vp, vp, ctypes.c_int32, vp, vp, vp, vp]
    lib.stream_check_device_status.restype = ctypes.c_int
    lib.stream_check_device_status.argtypes = [vp]
    lib.stream_host_staging_bytes.restype = sz
    lib.stream_host_staging_bytes.argtypes = [P]
    lib.stream_run_host.restype = ctypes.c_int
    lib.stream_run_host.argtypes = [P, vp, vp, vp, vp, vp, ctypes.c_float, vp, sz, vp]
    lib.stream_run_host_var.restype = ctypes.c_int
    lib.stream_run_host_var.argtypes = [P, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, sz, vp]
    PC, i32, i64 = ctypes.POINTER(StreamCache), ctypes.c_int32, ctypes.c_int64
    lib.stream_prompt_attention.restype = ctypes.c_int
    lib.stream_prompt_attention.argtypes = [vp, vp,  # (the struct, or its bytes)
                                             vp, vp, vp, vp, ctypes.c_float, vp, vp, vp]
    lib.stream_cache_workspace_bytes.restype = sz
    lib.stream_cache_workspace_bytes.argtypes = [PC]
    lib.stream_cache_reserve.restype = ctypes.c_int
    lib.stream_cache_reserve.argtypes = [PC, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.stream_cache_fork.restype = ctypes.c_int
    lib.stream_cache_fork.argtypes = [PC, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.stream_cache_free.restype = ctypes.c_int
    lib.stream_cache_free.argtypes = [PC, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.stream_cache_compact.restype = ctypes.c_int
    lib.stream_cache_compact.argtypes = [PC, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.stream_cache_copy_pages.restype = ctypes.c_int
    lib.stream_cache_copy_pages.argtypes = [PC, vp, vp, vp, vp, i32, vp]
    lib.stream_cache_write.restype = ctypes.c_int
    lib.stream_cache_write.argtypes = [PC, i32, vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.stream_decode_workspace_bytes.restype = sz
    lib.stream_decode_workspace_bytes.argtypes = [PC, i32]
    lib.stream_decode_attention.restype = ctypes.c_int
    lib.stream_decode_attention.argtypes = [PC, i32, i32, vp, i64, i64, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, sz, vp]
    P8 = ctypes.POINTER(StreamCache8)
    lib.stream_cache_read.restype = ctypes.c_int
    lib.stream_cache_read.argtypes = [PC, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp]
    lib.stream_prompt_window_attention.restype = ctypes.c_int
    lib.stream_prompt_window_attention.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp]
    lib.stream_decode_window_attention.restype = ctypes.c_int
    lib.stream_decode_window_attention.argtypes = [PC, i32, i32, i32, i32, vp, i64, i64, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, sz, vp]
    lib.stream_cache8_write.restype = ctypes.c_int
    lib.stream_cache8_write.argtypes = [P8, i32, vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.stream_cache8_read.restype = ctypes.c_int
    lib.stream_cache8_read.argtypes = [P8, i32, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp]
    lib.stream_cache8_copy_pages.restype = ctypes.c_int
    lib.stream_cache8_copy_pages.argtypes = [P8, vp, vp, vp, vp, vp, vp, i32, vp]
    lib.stream_decode_attention8.restype = ctypes.c_int
    lib.stream_decode_attention8.argtypes = [P8, i32, i32, i32, i32, vp, i64, i64, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, sz, vp]
    _lib = lib
    return lib


def _addr(x):
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    return None if x is None else int(x)


try:  # the current stream by its handle: a Stream object for it takes 3 us to make
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _current_device
except ImportError:  # (torch does not promise these names)
    _raw_stream = None


def _stream_handle(stream) -> int:
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        if not torch.cuda.is_initialized():
            torch.cuda.init()
        return _raw_stream(_current_device())
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


def _raise(status: int):
    if status:
        raise StreamError(status, _load().stream_last_error().decode())


# ----------------------------------------------------------------------------------------------
# One-to-one with the C ABI
# ----------------------------------------------------------------------------------------------
def stream_version() -> int:
    return int(_load().stream_version())


def stream_last_error() -> str:
    return _load().stream_last_error().decode()


def stream_workspace_bytes(p: StreamProblem) -> int:
    return int(_load().stream_workspace_bytes(ctypes.byref(p)))


def stream_build_mask(p: StreamProblem, q, k, mask_out, score_out, workspace, workspace_bytes: int, stream=None) -> None:
    _raise(_load().stream_build_mask(ctypes.byref(p), _addr(q), _addr(k), _addr(mask_out), _addr(score_out),
                                     _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_build_mask_var(p: StreamProblem, q, k, k_row, mask_out, score_out, workspace, workspace_bytes: int,
                          stream=None) -> None:
    """Mask build with ``k = k_row[query block]`` (device int32 array) instead of one k."""
    _raise(_load().stream_build_mask_var(ctypes.byref(p), _addr(q), _addr(k), _addr(k_row), _addr(mask_out),
                                         _addr(score_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_workspace_bytes_multi(p: StreamProblem, n_k: int) -> int:
    """Workspace with which a several-k build scores every (row, block) tile once (0 = invalid)."""
    return int(_load().stream_workspace_bytes_multi(ctypes.byref(p), int(n_k)))


def stream_build_mask_multi(p: StreamProblem, q, k, n_k: int, k_list_host, mask_out, score_out, workspace,
                            workspace_bytes: int, stream=None) -> None:
    """Masks for the ``n_k`` sparsity constants in the HOST int32 array ``k_list_host``, one slab each."""
    _raise(_load().stream_build_mask_multi(ctypes.byref(p), _addr(q), _addr(k), int(n_k), _addr(k_list_host),
                                           _addr(mask_out), _addr(score_out), _addr(workspace), workspace_bytes,
                                           _stream_handle(stream)))


def stream_k_schedule(p: StreamProblem, s: float, k_row_host) -> None:
    """Fills the HOST int32 array ``k_row_host`` ([ceil(T / block_q)]) with the per-row k for sparsity ``s``."""
    _raise(_load().stream_k_schedule(ctypes.byref(p), float(s), _addr(k_row_host)))


def stream_effective_k(T: int, block_q: int, s: float) -> int:
    """k for an effective sparsity ``s`` (the printed formula of Section 4.2, computed by the library)."""
    out = ctypes.c_int32(0)
    _raise(_load().stream_effective_k(int(T), int(block_q), float(s), ctypes.byref(out)))
    return int(out.value)


def stream_selftest_bounded_wait(limit_cycles: int, workspace, workspace_bytes: int, stream=None) -> None:
    """Diagnostic kernel whose bounded wait runs out after ``limit_cycles``; read the outcome with stream_read_stats."""
    _raise(_load().stream_selftest_bounded_wait(int(limit_cycles), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_probe_scratch_bytes() -> int:
    return int(_load().stream_probe_scratch_bytes())


def stream_probe_unit_rates(scratch, scratch_bytes: int, stream=None) -> StreamUnitRates:
    out = StreamUnitRates()
    _raise(_load().stream_probe_unit_rates(_addr(scratch), scratch_bytes, ctypes.byref(out), _stream_handle(stream)))
    return out


def stream_build_mask_static(p: StreamProblem, q, k, mask_out, score_out, stream=None) -> None:
    """Mask build on the library's built-in scratch: no workspace argument, nothing allocated."""
    _raise(_load().stream_build_mask_static(ctypes.byref(p), _addr(q), _addr(k), _addr(mask_out), _addr(score_out),
                                            _stream_handle(stream)))


def stream_sparse_attention(p: StreamProblem, q, k, v, mask, scale: float, out, stream=None) -> None:
    _raise(_load().stream_sparse_attention(ctypes.byref(p), _addr(q), _addr(k), _addr(v), _addr(mask), float(scale),
                                           _addr(out), _stream_handle(stream)))


def stream_read_stats(workspace, stream=None) -> StreamStats:
    st = StreamStats()
    _raise(_load().stream_read_stats(_addr(workspace), ctypes.byref(st), _stream_handle(stream)))
    return st


def stream_vertical_scores(p: StreamProblem, mask, scores, vertical_out, kurtosis_out, workspace, workspace_bytes: int,
                           stream=None) -> None:
    _raise(_load().stream_vertical_scores(ctypes.byref(p), _addr(mask), _addr(scores), _addr(vertical_out),
                                          _addr(kurtosis_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_mask_difference(n_rows: int, k_a: int, mask_a, scores_a, k_b: int, mask_b, diff_out, diff_scores_out, stream=None) -> None:
    _raise(_load().stream_mask_difference(n_rows, k_a, _addr(mask_a), _addr(scores_a), k_b, _addr(mask_b), _addr(diff_out),
                                          _addr(diff_scores_out), _stream_handle(stream)))


def stream_check_device_status(stream=None) -> None:
    """Drains the stream; raises if a kernel without a workspace recorded a bounded wait that ran out."""
    _raise(_load().stream_check_device_status(_stream_handle(stream)))


def stream_host_staging_bytes(p: StreamProblem) -> int:
    return int(_load().stream_host_staging_bytes(ctypes.byref(p)))


def stream_run_host(p: StreamProblem, q_host, k_host, v_host, mask_host, out_host, scale: float, staging,
                    staging_bytes: int, stream=None) -> None:
    _raise(_load().stream_run_host(ctypes.byref(p), _addr(q_host), _addr(k_host), _addr(v_host), _addr(mask_host),
                                   _addr(out_host), float(scale), _addr(staging), staging_bytes, _stream_handle(stream)))


def stream_run_host_var(p: StreamProblem, q_host, k_host, v_host, k_row_host, mask_host, out_host, scale: float, staging,
                        staging_bytes: int, stream=None) -> None:
    """The host path with one k per query block (``k_row_host``: HOST int32 array)."""
    _raise(_load().stream_run_host_var(ctypes.byref(p), _addr(q_host), _addr(k_host), _addr(v_host), _addr(k_row_host),
                                       _addr(mask_host), _addr(out_host), float(scale), _addr(staging), staging_bytes,
                                       _stream_handle(stream)))


def stream_prompt_attention(p: StreamPrompt, q, k, v, cu_q, cu_k, scale: float, out, lse_out, stream=None) -> None:
    """Dense attention of packed prompts."""
    _raise(_load().stream_prompt_attention(ctypes.byref(p), _addr(q), _addr(k), _addr(v), _addr(cu_q), _addr(cu_k), float(scale),
                                           _addr(out), _addr(lse_out), _stream_handle(stream)))


def stream_cache_workspace_bytes(c: StreamCache) -> int:
    return int(_load().stream_cache_workspace_bytes(ctypes.byref(c)))


def stream_cache_reserve(c: StreamCache, n_new, page_table, seq_len, ref_count, info_out, workspace, workspace_bytes: int, stream=None) -> None:
    _raise(_load().stream_cache_reserve(ctypes.byref(c), _addr(n_new), _addr(page_table), _addr(seq_len), _addr(ref_count),
                                        _addr(info_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_cache_fork(c: StreamCache, parent, page_table, seq_len, ref_count, pairs_out, info_out, workspace, workspace_bytes: int,
                      stream=None) -> None:
    _raise(_load().stream_cache_fork(ctypes.byref(c), _addr(parent), _addr(page_table), _addr(seq_len), _addr(ref_count),
                                     _addr(pairs_out), _addr(info_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_cache_free(c: StreamCache, done, page_table, seq_len, ref_count, info_out, workspace, workspace_bytes: int, stream=None) -> None:
    _raise(_load().stream_cache_free(ctypes.byref(c), _addr(done), _addr(page_table), _addr(seq_len), _addr(ref_count),
                                     _addr(info_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_cache_compact(c: StreamCache, page_table, seq_len, ref_count, pairs_out, info_out, workspace, workspace_bytes: int,
                         stream=None) -> None:
    _raise(_load().stream_cache_compact(ctypes.byref(c), _addr(page_table), _addr(seq_len), _addr(ref_count), _addr(pairs_out),
                                        _addr(info_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_cache_copy_pages(c: StreamCache, k_pages, v_pages, pairs, count, n_pairs: int, stream=None) -> None:
    _raise(_load().stream_cache_copy_pages(ctypes.byref(c), _addr(k_pages), _addr(v_pages), _addr(pairs), _addr(count), int(n_pairs),
                                           _stream_handle(stream)))


def stream_cache_write(c: StreamCache, layer: int, k, v, total: int, stride_t: int, stride_h: int, cu_new, page_table, seq_len,
                       done, k_pages, v_pages, stream=None) -> None:
    _raise(_load().stream_cache_write(ctypes.byref(c), int(layer), _addr(k), _addr(v), int(total), int(stride_t), int(stride_h),
                                      _addr(cu_new), _addr(page_table), _addr(seq_len), _addr(done), _addr(k_pages), _addr(v_pages),
                                      _stream_handle(stream)))


def stream_decode_workspace_bytes(c: StreamCache, n_q_heads: int) -> int:
    return int(_load().stream_decode_workspace_bytes(ctypes.byref(c), int(n_q_heads)))


def stream_decode_attention(c: StreamCache, layer: int, n_q_heads: int, q, q_stride_s: int, q_stride_h: int, k_pages, v_pages,
                            page_table, seq_len, scale: float, out, lse_out, workspace, workspace_bytes: int, stream=None) -> None:
    """Attention of one new token of every slot over a paged cache."""
    _raise(_load().stream_decode_attention(ctypes.byref(c), int(layer), int(n_q_heads), _addr(q), int(q_stride_s), int(q_stride_h),
                                           _addr(k_pages), _addr(v_pages), _addr(page_table), _addr(seq_len), float(scale),
                                           _addr(out), _addr(lse_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_cache_read(c: StreamCache, layer: int, k_pages, v_pages, cu, total: int, page_table, seq_len, k_out, v_out, stream=None) -> None:
    _raise(_load().stream_cache_read(ctypes.byref(c), layer, _addr(k_pages), _addr(v_pages), _addr(cu), total, _addr(page_table), _addr(seq_len),
                                     _addr(k_out), _addr(v_out), _stream_handle(stream)))


def stream_prompt_window_attention(p: StreamPrompt, window: int, sinks: int, q, k, v, cu_q, cu_k, scale: float, out, lse_out, stream=None) -> None:
    _raise(_load().stream_prompt_window_attention(ctypes.byref(p), window, sinks, _addr(q), _addr(k), _addr(v), _addr(cu_q), _addr(cu_k), scale,
                                                  _addr(out), _addr(lse_out), _stream_handle(stream)))


def stream_decode_window_attention(c: StreamCache, layer: int, n_q_heads: int, window: int, sinks: int, q, q_stride_s: int, q_stride_h: int, k_pages,
                                   v_pages, page_table, seq_len, scale: float, out, lse_out, workspace, workspace_bytes: int, stream=None) -> None:
    _raise(_load().stream_decode_window_attention(ctypes.byref(c), layer, n_q_heads, window, sinks, _addr(q), q_stride_s, q_stride_h, _addr(k_pages),
                                                  _addr(v_pages), _addr(page_table), _addr(seq_len), scale, _addr(out), _addr(lse_out),
                                                  _addr(workspace), workspace_bytes, _stream_handle(stream)))


def stream_cache8_write(c: StreamCache8, layer: int, k, v, total: int, stride_t: int, stride_h: int, cu_new, page_table, seq_len, done, k_pages,
                        v_pages, k_scale, v_scale, stream=None) -> None:
    _raise(_load().stream_cache8_write(ctypes.byref(c), layer, _addr(k), _addr(v), total, stride_t, stride_h, _addr(cu_new), _addr(page_table),
                                       _addr(seq_len), _addr(done), _addr(k_pages), _addr(v_pages), _addr(k_scale), _addr(v_scale),
                                       _stream_handle(stream)))


def stream_cache8_read(c: StreamCache8, layer: int, k_pages, v_pages, k_scale, v_scale, cu, total: int, page_table, seq_len, k_out, v_out,
                       stream=None) -> None:
    _raise(_load().stream_cache8_read(ctypes.byref(c), layer, _addr(k_pages), _addr(v_pages), _addr(k_scale), _addr(v_scale), _addr(cu), total,
                                      _addr(page_table), _addr(seq_len), _addr(k_out), _addr(v_out), _stream_handle(stream)))


def stream_cache8_copy_pages(c: StreamCache8, k_pages, v_pages, k_scale, v_scale, pairs, count, n_pairs: int, stream=None) -> None:
    _raise(_load().stream_cache8_copy_pages(ctypes.byref(c), _addr(k_pages), _addr(v_pages), _addr(k_scale), _addr(v_scale), _addr(pairs), _addr(count),
                                            n_pairs, _stream_handle(stream)))


def stream_decode_attention8(c: StreamCache8, layer: int, n_q_heads: int, window: int, sinks: int, q, q_stride_s: int, q_stride_h: int, k_pages,
                             v_pages, k_scale, v_scale, page_table, seq_len, scale: float, out, lse_out, workspace, workspace_bytes: int,
                             stream=None) -> None:
    _raise(_load().stream_decode_attention8(ctypes.byref(c), layer, n_q_heads, window, sinks, _addr(q), q_stride_s, q_stride_h, _addr(k_pages),
                                            _addr(v_pages), _addr(k_scale), _addr(v_scale), _addr(page_table), _addr(seq_len), scale, _addr(out),
                                            _addr(lse_out), _addr(workspace), workspace_bytes, _stream_handle(stream)))


# ----------------------------------------------------------------------------------------------
# Conveniences: problem struct from tensors, outputs allocated with torch
# ----------------------------------------------------------------------------------------------
def make_problem(q: torch.Tensor, k: torch.Tensor, *, block_q: int, block_k: int, k_top: int, causal: bool = True,
                 impl: str = "auto") -> StreamProblem:
    """Problem struct for q ``[B, H, T, d]`` and k ``[B, G, T, d]`` (any strides with unit innermost)."""
    qs, ks, dtype = q.shape, k.shape, q.dtype
    if len(qs) != 4 or len(ks) != 4 or qs[0] != ks[0] or qs[2] != ks[2] or qs[3] != ks[3]:
        raise ValueError("q must be [B, H, T, d] and k [B, G, T, d] with matching B, T, d")
    if k.dtype is not dtype or (dtype is not torch.float32 and dtype is not torch.bfloat16):
        raise ValueError("q and k must both be float32 or bfloat16")
    (q_b, q_h, q_t, q_d), (k_b, k_h, k_t, k_d) = q.stride(), k.stride()
    if q_d != 1 or k_d != 1:
        raise ValueError("innermost stride must be 1")
    fields = (qs[0], qs[1], ks[1], qs[2], qs[3], block_q, block_k, k_top, int(causal),
              STREAM_F32 if dtype is torch.float32 else STREAM_BF16, IMPL[impl], q_b, q_h, q_t, k_b, k_h, k_t)
    try:  # (packed at once: field by field the struct takes three times as long)
        return StreamProblem.from_buffer_copy(_PROBLEM.pack(*fields))
    except struct.error:  # not whole numbers, or none that fit: as ctypes takes them
        return StreamProblem(*fields)


def n_query_blocks(p: StreamProblem) -> int:
    return -(-p.T // p.block_q)


@dataclass
class MaskResult:
    mask: torch.Tensor            # int32 [B, H, n_query_blocks, k_top]
    scores: torch.Tensor | None   # float32, same shape, if requested
    workspace: torch.Tensor       # holds the counters of this call; see stream_read_stats
    header_bytes: int = 256       # stream_workspace_bytes of the problem: optional per-row counters sit behind it

    def stats(self, stream=None) -> StreamStats:
        return stream_read_stats(self.workspace, stream)

    def row_tiles(self) -> torch.Tensor | None:
        """int32 [B, H, n_query_blocks]: tiles scored per row, if the workspace had room for them."""
        rows = self.mask.shape[0] * self.mask.shape[1] * self.mask.shape[2]
        if self.mask.dim() != 4 or self.workspace.numel() < self.header_bytes + 4 * rows:
            return None
        return self.workspace[self.header_bytes:self.header_bytes + 4 * rows].view(torch.int32).view(self.mask.shape[:3])


def _empty(shape, dtype, device) -> torch.Tensor:
    """Contiguous new tensor (with its strides given, it costs a third less of the host's time)."""
    strides, n = [1] * len(shape), 1
    for i in range(len(shape) - 1, -1, -1):
        strides[i] = n
        n *= max(1, shape[i])
    return torch.empty_strided(shape, strides, dtype=dtype, device=device)


def _header_bytes(p: StreamProblem) -> int:
    n = (_lib or _load()).stream_workspace_bytes(ctypes.byref(p))
    if n == 0:
        raise StreamError(STREAM_ERR_INVALID_ARG, stream_last_error())
    return n


def new_workspace(p: StreamProblem, device, row_tiles: bool = False) -> torch.Tensor:
    """Workspace of the size the library asks for; with ``row_tiles`` also room for one counter per row."""
    n = _header_bytes(p)
    if row_tiles:
        n += 4 * p.batch * p.n_q_heads * n_query_blocks(p)
    return torch.empty(n, dtype=torch.uint8, device=device)


def build_mask(q: torch.Tensor, k: torch.Tensor, *, block_q: int, block_k: int, k_top: int, causal: bool = True,
               impl: str = "auto", want_scores: bool = False, mask_out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None, k_row: torch.Tensor | None = None, row_tiles: bool = False,
               stream=None) -> MaskResult:
    """Mask of every row. With ``k_row`` (int32 CUDA tensor, one k per query block, see
    :func:`k_schedule`) each row uses its own k and ``k_top`` is the row width. ``row_tiles``
    makes the workspace large enough for the per-row tile counters (``MaskResult.row_tiles()``)."""
    if not q.is_cuda or not k.is_cuda:
        raise ValueError("q and k must be CUDA tensors (there is no CPU path)")
    p = make_problem(q, k, block_q=block_q, block_k=block_k, k_top=k_top, causal=causal, impl=impl)
    header = _header_bytes(p) if workspace is None else 0  # (with a workspace the call itself says what is wrong with the problem)
    device, shape = q.device, (p.batch, p.n_q_heads, n_query_blocks(p), k_top)
    mask = mask_out if mask_out is not None else _empty(shape, torch.int32, device)
    scores = _empty(shape, torch.float32, device) if want_scores else None
    if workspace is None:
        workspace = _empty((header + (4 * shape[0] * shape[1] * shape[2] if row_tiles else 0),), torch.uint8, device)
    if k_row is None:
        stream_build_mask(p, q, k, mask, scores, workspace, workspace.numel(), stream)
    else:
        if not k_row.is_cuda or k_row.dtype != torch.int32 or not k_row.is_contiguous() or tuple(k_row.shape) != (shape[2],):
            raise ValueError(f"k_row must be a contiguous int32 CUDA tensor of shape ({shape[2]},)")
        stream_build_mask_var(p, q, k, k_row, mask, scores, workspace, workspace.numel(), stream)
    return MaskResult(mask, scores, workspace, header or _header_bytes(p))


def build_masks(q: torch.Tensor, k: torch.Tensor, k_list, *, block_q: int, block_k: int, causal: bool = True,
                impl: str = "auto", want_scores: bool = False, share: bool = True, stream=None) -> MaskResult:
    """Masks for every k in ``k_list`` in one call: ``mask`` is [len(k_list), B, H, rows, max(k_list)].
    ``share=False`` gives the library only the small workspace (the tensor-core kernel then runs
    once per k and does not reuse tile scores between them)."""
    if not q.is_cuda or not k.is_cuda:
        raise ValueError("q and k must be CUDA tensors (there is no CPU path)")
    ks = array.array("i", [int(x) for x in k_list])  # (an entry beyond 32 bits is an error)
    p = make_problem(q, k, block_q=block_q, block_k=block_k, k_top=max(ks), causal=causal, impl=impl)
    shape = (len(ks), p.batch, p.n_q_heads, n_query_blocks(p), p.k_top)
    mask = _empty(shape, torch.int32, q.device)
    scores = _empty(shape, torch.float32, q.device) if want_scores else None
    n_ws = stream_workspace_bytes_multi(p, len(ks)) if share else stream_workspace_bytes(p)
    if n_ws == 0:
        raise StreamError(STREAM_ERR_INVALID_ARG, stream_last_error())
    ws = _empty((n_ws,), torch.uint8, q.device)
    stream_build_mask_multi(p, q, k, len(ks), ks.buffer_info()[0], mask, scores, ws, n_ws, stream)
    return MaskResult(mask, scores, ws)


def k_schedule(p: StreamProblem, s: float) -> torch.Tensor:
    """Host int32 tensor [ceil(T / block_q)]: k per query block for an effective sparsity ``s``
    (the formula of :func:`effective_k` applied to each row's own number of allowed key blocks,
    clamped to ``1 .. p.k_top``). Move it to the device for :func:`build_mask`."""
    out = torch.empty((n_query_blocks(p),), dtype=torch.int32)
    stream_k_schedule(p, s, out.data_ptr())
    return out


def sparse_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, mask: torch.Tensor, *, block_q: int,
                     block_k: int, causal: bool = True, scale: float = 0.0, impl: str = "auto",
                     out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    if not (q.is_cuda and k.is_cuda and v.is_cuda and mask.is_cuda):
        raise ValueError("q, k, v and mask must be CUDA tensors (there is no CPU path)")
    if v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype:
        raise ValueError("v must have k's shape, strides and dtype")
    if mask.dtype != torch.int32 or not mask.is_contiguous():
        raise ValueError("mask must be a contiguous int32 tensor")
    m_shape = tuple(mask.shape)
    p = make_problem(q, k, block_q=block_q, block_k=block_k, k_top=m_shape[-1], causal=causal, impl=impl)
    B, H, T, d = q.shape
    if m_shape != (B, H, -(-T // block_q), m_shape[-1]):
        raise ValueError("mask must be [B, H, ceil(T / block_q), k_top]")
    if out is None:
        out = _empty((B, H, T, d), q.dtype, q.device)
    stream_sparse_attention(p, q, k, v, mask, scale, out, stream)
    return out


def run_host(q_host: torch.Tensor, k_host: torch.Tensor, v_host: torch.Tensor, mask_host: torch.Tensor,
             out_host: torch.Tensor, staging: torch.Tensor, *, block_q: int, block_k: int, k_top: int,
             causal: bool = True, scale: float = 0.0, impl: str = "auto", k_row: torch.Tensor | None = None, stream=None) -> None:
    """Whole path from (pinned) host tensors through a caller-provided device staging buffer. With
    ``k_row`` (HOST int32 tensor, one k per query block) the mask is the variable-k build."""
    if q_host.is_cuda or not staging.is_cuda:
        raise ValueError("q/k/v/mask/out live on the host, staging on the device")
    p = make_problem(q_host, k_host, block_q=block_q, block_k=block_k, k_top=k_top, causal=causal, impl=impl)
    if k_row is None:
        stream_run_host(p, q_host, k_host, v_host, mask_host, out_host, scale, staging, staging.numel(), stream)
    else:
        if k_row.is_cuda or k_row.dtype != torch.int32 or not k_row.is_contiguous() or k_row.numel() != n_query_blocks(p):
            raise ValueError("k_row must be a contiguous int32 HOST tensor with one entry per query block")
        stream_run_host_var(p, q_host, k_host, v_host, k_row, mask_host, out_host, scale, staging, staging.numel(), stream)


def vertical_scores(p: StreamProblem, mask: torch.Tensor, scores: torch.Tensor | None = None, stream=None):
    """(vertical [B, H, ceil(T / block_k)], kurtosis [B, H]) of a mask, binary or weighted by ``scores``."""
    if not mask.is_cuda or mask.dtype != torch.int32 or not mask.is_contiguous():
        raise ValueError("mask must be a contiguous int32 CUDA tensor")
    if scores is not None and (scores.shape != mask.shape or scores.dtype != torch.float32 or not scores.is_contiguous()):
        raise ValueError("scores must be a contiguous float32 tensor of the mask's shape")
    n_kb = -(-p.T // p.block_k)
    vert = _empty((p.batch, p.n_q_heads, n_kb), torch.float32, mask.device)
    kurt = _empty((p.batch, p.n_q_heads), torch.float32, mask.device)
    ws = new_workspace(p, mask.device)
    stream_vertical_scores(p, mask, scores, vert, kurt, ws, ws.numel(), stream)
    stream_read_stats(ws, stream)
    return vert, kurt


def mask_difference(mask_a: torch.Tensor, mask_b: torch.Tensor, scores_a: torch.Tensor | None = None, stream=None):
    """Row-wise ``mask_a`` minus ``mask_b`` (same leading shape, last dims k_a and k_b); returns (diff, scores or None)."""
    if mask_a.shape[:-1] != mask_b.shape[:-1] or mask_a.dtype != torch.int32 or mask_b.dtype != torch.int32:
        raise ValueError("masks must be int32 with the same leading shape")
    if not (mask_a.is_cuda and mask_b.is_cuda and mask_a.is_contiguous() and mask_b.is_contiguous()):
        raise ValueError("masks must be contiguous CUDA tensors")
    if scores_a is not None and (scores_a.shape != mask_a.shape or scores_a.dtype != torch.float32 or not scores_a.is_contiguous()):
        raise ValueError("scores_a must be a contiguous float32 tensor of mask_a's shape")
    diff = torch.empty_like(mask_a)
    dsc = torch.empty_like(scores_a) if scores_a is not None else None
    n = mask_a.numel() // mask_a.shape[-1]
    stream_mask_difference(n, mask_a.shape[-1], mask_a, scores_a, mask_b.shape[-1], mask_b, diff, dsc, stream)
    return diff, dsc


def effective_k(T: int, block_q: int, s: float) -> int:
    """Sparsity constant for an effective sparsity ``s`` in [0, 1] (Section 4.2 of the paper), as
    computed by the library's ``stream_effective_k``."""
    return stream_effective_k(T, block_q, s)


def probe_unit_rates(device="cuda", stream=None) -> StreamUnitRates:
    """TMA gather rate and tensor-core instruction time of the current device (``stream_probe_unit_rates``)."""
    n = stream_probe_scratch_bytes()
    if n == 0:
        raise RuntimeError("no CUDA device to probe")
    scratch = torch.empty(n, dtype=torch.uint8, device=device)
    return stream_probe_unit_rates(scratch, n, stream)


# ----------------------------------------------------------------------------------------------
# Dense attention and the paged cache
# ----------------------------------------------------------------------------------------------
_DTYPES = {torch.float32: STREAM_F32, torch.bfloat16: STREAM_BF16}


def _checked(x: torch.Tensor, dtype, shape, what: str, device) -> torch.Tensor:
    if x.dtype is not dtype or not x.is_contiguous() or x.shape != shape or x.device != device:
        raise ValueError(f"{what} must be a contiguous {str(dtype)[6:]} tensor of shape {tuple(shape)} on {device}")
    return x


def _launch(device: torch.device, call, args, stream) -> None:
    """``call(*args, stream)`` with the tensors' device as the current one (the way to another device and back is taken
    only where it is another; of the host's time a short call takes, half is argument handling)."""
    if device.index == (torch.cuda.current_device() if _raw_stream is None else _current_device()):
        status = call(*args, _stream_handle(stream))
    else:
        with torch.cuda.device(device):
            status = call(*args, _stream_handle(stream))
    if status:
        _raise(status)


def _checked_stream(stream, device: torch.device):
    """A stream, or its handle, of whose device nothing is known."""
    if isinstance(stream, torch.cuda.Stream) and stream.device != device:
        raise ValueError("the stream must be one of the tensors' device")
    return stream


def _on_stream(stream, device: torch.device, call, *args, **kwargs):
    """``call`` with ``stream`` as the current one: what it allocates is then that stream's memory, which nobody on another
    one is given while the kernels have yet to run (a workspace is let go when the call returns)."""
    if not isinstance(_checked_stream(stream, device), torch.cuda.Stream):
        handle = int(stream)
        stream = torch.cuda.ExternalStream(handle, device=device) if handle > 1 else torch.cuda.default_stream(device)  # (1: cudaStreamLegacy)
    with torch.cuda.stream(stream):
        return call(*args, **kwargs)


_PROMPT = struct.Struct("@iiiiqqiiqqqq")  # StreamPrompt's fields
assert _PROMPT.size == ctypes.sizeof(StreamPrompt)


def _window(window: int, sinks: int) -> tuple[int, int]:
    """As the library takes them: larger than any sequence is as large as any."""
    if window < 0 or sinks < 0:
        raise ValueError("window and sinks must not be negative")
    if sinks and not window:
        raise ValueError("sinks are what is seen beside a window")
    return min(window, 0x7fffffff), min(sinks, 0x7fffffff)


def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor | None = None, *,
                     causal: bool = True, scale: float = 0.0, window: int = 0, sinks: int = 0, want_lse: bool = False,
                     out: torch.Tensor | None = None, lse_out: torch.Tensor | None = None, stream=None):
    """Dense attention of packed prompts: q ``[total_q, H, d]``, k and v ``[total_k, G, d]``, ``cu_q`` and ``cu_k``
    int32 CUDA tensors ``[n_seqs + 1]`` with the sequences' first rows (``cu_k``: default ``cu_q``). Under a causal
    mask a sequence's last query sees all its keys; with a ``window`` (0: none) a query sees the last ``window`` of those keys, its own among
    them, and the first ``sinks``. Returns the output ``[total_q, H, d]``, with ``want_lse`` (or
    ``lse_out``) also the logarithms of the softmax sums, float32 ``[H, total_q]``. Rows of no sequence are left as they are. ``stream``, here and
    below: the call runs and allocates as under ``torch.cuda.stream(stream)``."""
    if not (q.is_cuda and k.is_cuda and v.is_cuda and cu_q.is_cuda):
        raise ValueError("q, k, v and cu_q must be CUDA tensors (there is no CPU path)")
    qs, ks, q_strides, k_strides, dtype, device = q.shape, k.shape, q.stride(), k.stride(), q.dtype, q.device
    if len(qs) != 3 or len(ks) != 3 or qs[2] != ks[2]:
        raise ValueError("q must be [total_q, H, d] and k [total_k, G, d]")
    if v.shape != ks or v.stride() != k_strides:
        raise ValueError("v must have k's shape and strides")
    if dtype not in _DTYPES or k.dtype is not dtype or v.dtype is not dtype:
        raise ValueError("q, k and v must all be float32 or all bfloat16")
    if q_strides[2] != 1 or k_strides[2] != 1:
        raise ValueError("innermost stride must be 1")
    if k.device != device or v.device != device:
        raise ValueError("q, k and v must be on one device")
    n = cu_q.shape
    if len(n) != 1 or n[0] < 2:
        raise ValueError("cu_q must be [n_seqs + 1]")
    _checked(cu_q, torch.int32, n, "cu_q", device)
    if cu_k is None:
        cu_k = cu_q
    elif cu_k is not cu_q:
        _checked(cu_k, torch.int32, n, "cu_k", device)
    if stream is not None:
        return _on_stream(stream, device, prompt_attention, q, k, v, cu_q, cu_k, causal=causal, scale=scale, window=window, sinks=sinks,
                          want_lse=want_lse, out=out, lse_out=lse_out)
    if window or sinks:
        window, sinks = _window(window, sinks)
        if not causal:
            raise ValueError("a window looks back: causal must be true")
    total, H, d = qs
    fields = (n[0] - 1, H, ks[1], d, total, ks[0], int(causal), _DTYPES[dtype], q_strides[0], q_strides[1], k_strides[0], k_strides[1])
    try:
        p = _PROMPT.pack(*fields)
    except struct.error:  # sizes beyond 32 bits: the library's to refuse
        p = ctypes.byref(StreamPrompt(*fields))
    if out is None:
        out = torch.empty_strided(qs, (H * d, d, 1), dtype=dtype, device=device)
    else:
        _checked(out, dtype, qs, "out", device)
    if lse_out is not None:
        _checked(lse_out, torch.float32, (H, total), "lse_out", device)
    elif want_lse:
        lse_out = torch.empty_strided((H, total), (total, 1), dtype=torch.float32, device=device)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), scale, out.data_ptr(),
            None if lse_out is None else lse_out.data_ptr())
    if window:
        _launch(device, (_lib or _load()).stream_prompt_window_attention, (p, window, sinks, *args), None)
    else:
        _launch(device, (_lib or _load()).stream_prompt_attention, (p, *args), None)
    return out if lse_out is None else (out, lse_out)


@dataclass
class CacheMoves:
    """Page copies that are due (:func:`cache_copy_pages`) and what the call that asks for them says of itself."""

    pairs: torch.Tensor  # int32 [n, 2]: {from, to}, then -1
    info: torch.Tensor   # int32 [4]: done, pages to copy, free pages, refusals


class PagedCache:
    """A paged key-value cache of one or several layers and its ledger; see ``stream_cache`` in stream.h.

    ``k`` and ``v`` are ``[n_layers, n_pages, page_size, n_kv_heads, d]`` (views of any stride order, innermost
    stride 1, both alike), ``page_table`` int32 ``[n_slots, max_pages]``, ``seq_len`` int32 ``[n_slots]`` and
    ``ref_count`` int32 ``[n_pages]``, all on one device. The object keeps them and nothing else on the device;
    :func:`new_cache` makes an empty one."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, seq_len: torch.Tensor, ref_count: torch.Tensor):
        if not k.is_cuda or not v.is_cuda:
            raise ValueError("k and v must be CUDA tensors (there is no CPU path)")
        if k.dim() != 5 or v.shape != k.shape or v.stride() != k.stride() or v.dtype is not k.dtype or v.device != k.device:
            raise ValueError("k and v must be [n_layers, n_pages, page_size, n_kv_heads, d], alike in strides, dtype and device")
        if k.dtype not in _DTYPES:
            raise ValueError("k and v must be float32 or bfloat16")
        self._keep(k, v, page_table, seq_len, ref_count, k.dtype)

    def _keep(self, k, v, page_table, seq_len, ref_count, dtype) -> None:
        if k.stride(4) != 1:
            raise ValueError("innermost stride must be 1")
        if page_table.dim() != 2:
            raise ValueError("page_table must be [n_slots, max_pages]")
        self.device = k.device
        self.n_layers, self.n_pages, self.page_size, self.n_kv_heads, self.d = k.shape
        self.n_slots, self.max_pages = page_table.shape
        self.k, self.v = k, v
        self.page_table = _checked(page_table, torch.int32, page_table.shape, "page_table", self.device)
        self.seq_len = _checked(seq_len, torch.int32, (self.n_slots,), "seq_len", self.device)
        self.ref_count = _checked(ref_count, torch.int32, (self.n_pages,), "ref_count", self.device)
        self.struct = StreamCache(self.n_slots, self.n_pages, self.page_size, self.max_pages, self.n_kv_heads, self.d, self.n_layers,
                                  _DTYPES[dtype], *k.stride()[:4])
        n = stream_cache_workspace_bytes(self.struct)
        if n == 0:
            raise StreamError(STREAM_ERR_INVALID_ARG, stream_last_error())
        self._ledger_bytes = n
        self._p = ctypes.byref(self.struct)
        self._decode_bytes = {}  # workspace of decode_attention by query heads

    @property
    def dtype(self) -> torch.dtype:
        """Of queries, outputs and new keys and values."""
        return self.k.dtype

    def _pages(self):
        return self.k.data_ptr(), self.v.data_ptr()

    def _ledger(self):
        return self.page_table.data_ptr(), self.seq_len.data_ptr(), self.ref_count.data_ptr()

    def _info(self):
        return torch.empty_strided((4,), (1,), dtype=torch.int32, device=self.device)

    def _workspace(self):
        """For one ledger call: the current stream's memory, as the call's results are. (The handle may be gone before the call has run, and
        a graph that the call is captured in outlives it.)"""
        return torch.empty_strided((self._ledger_bytes,), (1,), dtype=torch.uint8, device=self.device)


class PagedCache8(PagedCache):
    """A paged key-value cache in 8 bits; see ``stream_cache8`` in stream.h.

    ``k`` and ``v`` are float8_e4m3fn, ``k_scale`` and ``v_scale`` float32 ``[n_layers, n_pages, page_size / block, n_kv_heads]`` (any positive
    strides, both alike): a key is its e4m3 numbers times its block's scale. ``dtype``: that of queries, outputs and new keys and values.
    The rest, and the ``cache_*`` functions and :func:`decode_attention`, as for :class:`PagedCache`; :func:`new_cache8` makes an empty one."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, page_table: torch.Tensor, seq_len: torch.Tensor,
                 ref_count: torch.Tensor, *, dtype: torch.dtype = torch.bfloat16):
        if not k.is_cuda or not v.is_cuda:
            raise ValueError("k and v must be CUDA tensors (there is no CPU path)")
        if k.dim() != 5 or v.shape != k.shape or v.stride() != k.stride() or v.device != k.device:
            raise ValueError("k and v must be [n_layers, n_pages, page_size, n_kv_heads, d], alike in strides and device")
        if k.dtype is not torch.float8_e4m3fn or v.dtype is not torch.float8_e4m3fn:
            raise ValueError("k and v must be float8_e4m3fn")
        if dtype not in _DTYPES:
            raise ValueError("dtype must be float32 or bfloat16")
        n, z = k.shape, k_scale.shape
        if len(z) != 4 or z[:2] != n[:2] or z[2] < 1 or n[2] % z[2] != 0 or z[3] != n[3]:
            raise ValueError("k_scale must be [n_layers, n_pages, page_size / block, n_kv_heads]")
        for x in (k_scale, v_scale):
            if x.dtype is not torch.float32 or x.device != k.device or x.shape != z or x.stride() != k_scale.stride():
                raise ValueError("k_scale and v_scale must be float32, alike, and on the device of k and v")
        self._keep(k, v, page_table, seq_len, ref_count, dtype)
        self.k_scale, self.v_scale, self.block = k_scale, v_scale, n[2] // z[2]
        self.struct8 = StreamCache8(self.struct, self.block, 0, *k_scale.stride())
        self._p8, self._dtype = ctypes.byref(self.struct8), dtype

    @property
    def dtype(self) -> torch.dtype:
        return self._dtype

    def _pages(self):
        return self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr()


def new_cache(n_slots: int, n_pages: int, page_size: int, max_pages: int, n_kv_heads: int, d: int, *, n_layers: int = 1,
              dtype: torch.dtype = torch.bfloat16, device="cuda") -> PagedCache:
    """An empty cache: all slots empty, all pages free (what the pages hold is not set)."""
    k, v = (torch.empty(n_layers, n_pages, page_size, n_kv_heads, d, dtype=dtype, device=device) for _ in range(2))
    return PagedCache(k, v, torch.full((n_slots, max_pages), -1, dtype=torch.int32, device=k.device),
                      torch.zeros(n_slots, dtype=torch.int32, device=k.device), torch.zeros(n_pages, dtype=torch.int32, device=k.device))


def new_cache8(n_slots: int, n_pages: int, page_size: int, max_pages: int, n_kv_heads: int, d: int, *, block: int, n_layers: int = 1,
               dtype: torch.dtype = torch.bfloat16, device="cuda") -> PagedCache8:
    """An empty cache in 8 bits whose tokens share a scale in blocks of ``block``, which divides ``page_size``. In memory a page has head after
    head: rows of 128 bytes that lie side by side are read faster than rows a token apart (four chains of up to 131072 tokens, 8 kv heads,
    d = 128: 52 us for 60)."""
    if block < 1 or page_size % block != 0:
        raise ValueError("block must be positive and divide page_size")
    k, v = (torch.empty(n_layers, n_pages, n_kv_heads, page_size, d, dtype=torch.float8_e4m3fn, device=device).transpose(2, 3) for _ in range(2))
    k_scale, v_scale = (torch.zeros(n_layers, n_pages, page_size // block, n_kv_heads, device=device) for _ in range(2))
    return PagedCache8(k, v, k_scale, v_scale, torch.full((n_slots, max_pages), -1, dtype=torch.int32, device=k.device),
                       torch.zeros(n_slots, dtype=torch.int32, device=k.device), torch.zeros(n_pages, dtype=torch.int32, device=k.device), dtype=dtype)


def cache_reserve(cache: PagedCache, n_new: torch.Tensor, stream=None) -> torch.Tensor:
    """Room for ``n_new`` (int32 ``[n_slots]``) more tokens in every slot, all of it or none; ``seq_len`` grows. Returns
    the info ``[done, pages taken, free pages, refusals]`` (int32, on the device)."""
    c = cache
    _checked(n_new, torch.int32, (c.n_slots,), "n_new", c.device)
    if stream is not None:
        return _on_stream(stream, c.device, cache_reserve, c, n_new)
    info, ws = c._info(), c._workspace()
    _launch(c.device, (_lib or _load()).stream_cache_reserve,
            (c._p, n_new.data_ptr(), *c._ledger(), info.data_ptr(), ws.data_ptr(), c._ledger_bytes), None)
    return info


def cache_fork(cache: PagedCache, parent: torch.Tensor, stream=None) -> CacheMoves:
    """Every slot s with ``parent[s] >= 0`` (int32 ``[n_slots]``) becomes a chain of its own with the tokens of slot
    ``parent[s]``. Full pages are shared; the copies of the others are due: hand the result to :func:`cache_copy_pages`."""
    c = cache
    _checked(parent, torch.int32, (c.n_slots,), "parent", c.device)
    if stream is not None:
        return _on_stream(stream, c.device, cache_fork, c, parent)
    info, ws, pairs = c._info(), c._workspace(), torch.empty_strided((c.n_slots, 2), (2, 1), dtype=torch.int32, device=c.device)
    _launch(c.device, (_lib or _load()).stream_cache_fork,
            (c._p, parent.data_ptr(), *c._ledger(), pairs.data_ptr(), info.data_ptr(), ws.data_ptr(), c._ledger_bytes), None)
    return CacheMoves(pairs, info)


def cache_free(cache: PagedCache, done: torch.Tensor, stream=None) -> torch.Tensor:
    """Empties every slot with ``done[s] != 0`` (int32 ``[n_slots]``). Returns ``[1, pages freed, free pages, impossible entries]``."""
    c = cache
    _checked(done, torch.int32, (c.n_slots,), "done", c.device)
    if stream is not None:
        return _on_stream(stream, c.device, cache_free, c, done)
    info, ws = c._info(), c._workspace()
    _launch(c.device, (_lib or _load()).stream_cache_free,
            (c._p, done.data_ptr(), *c._ledger(), info.data_ptr(), ws.data_ptr(), c._ledger_bytes), None)
    return info


def cache_compact(cache: PagedCache, stream=None) -> CacheMoves:
    """Moves the pages in use to the lowest numbers; the copies are due (:func:`cache_copy_pages`)."""
    c = cache
    if stream is not None:
        return _on_stream(stream, c.device, cache_compact, c)
    info, ws, pairs = c._info(), c._workspace(), torch.empty_strided((c.n_pages // 2, 2), (2, 1), dtype=torch.int32, device=c.device)
    _launch(c.device, (_lib or _load()).stream_cache_compact,
            (c._p, *c._ledger(), pairs.data_ptr(), info.data_ptr(), ws.data_ptr(), c._ledger_bytes), None)
    return CacheMoves(pairs, info)


def cache_copy_pages(cache: PagedCache, moves: CacheMoves, stream=None) -> None:
    """Makes the copies that :func:`cache_fork` or :func:`cache_compact` asks for, in all layers."""
    c, pairs, info = cache, moves.pairs, moves.info
    n = pairs.shape[0]
    _checked(pairs, torch.int32, (n, 2), "pairs", c.device)
    _checked(info, torch.int32, (4,), "info", c.device)
    args = *c._pages(), pairs.data_ptr(), info.data_ptr() + 4, n
    if isinstance(c, PagedCache8):
        _launch(c.device, (_lib or _load()).stream_cache8_copy_pages, (c._p8, *args), _checked_stream(stream, c.device))
    else:
        _launch(c.device, (_lib or _load()).stream_cache_copy_pages, (c._p, *args), _checked_stream(stream, c.device))


def cache_write(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, cu_new: torch.Tensor, *, layer: int = 0,
                info: torch.Tensor | None = None, stream=None) -> None:
    """Writes new tokens' keys and values (``[total, n_kv_heads, d]``, rows ``cu_new[s] .. cu_new[s + 1]`` being slot s's
    last tokens) to the pages of one layer, after :func:`cache_reserve`. With its ``info`` nothing is written if it was
    refused; a caller that has not looked at the info passes it on (the lengths are then as they were, and the last
    tokens there would be overwritten). A cache in 8 bits takes them rounded, and their blocks' scales."""
    c, shape, strides = cache, k.shape, k.stride()
    if len(shape) != 3 or shape[1] != c.n_kv_heads or shape[2] != c.d or v.shape != shape or v.stride() != strides:
        raise ValueError("k and v must be [total, n_kv_heads, d], alike in strides")
    if k.dtype is not c.dtype or v.dtype is not c.dtype or k.device != c.device or v.device != c.device:
        raise ValueError("k and v must have the cache's dtype and device")
    if strides[2] != 1:
        raise ValueError("innermost stride must be 1")
    _checked(cu_new, torch.int32, (c.n_slots + 1,), "cu_new", c.device)
    if info is not None:
        _checked(info, torch.int32, (4,), "info", c.device)
    if not 0 <= layer < c.n_layers:  # (beyond 32 bits too, of which the call would see the lower ones)
        raise ValueError("no such layer")
    args = (layer, k.data_ptr(), v.data_ptr(), shape[0], strides[0], strides[1], cu_new.data_ptr(), c.page_table.data_ptr(),
            c.seq_len.data_ptr(), None if info is None else info.data_ptr(), *c._pages())
    if isinstance(c, PagedCache8):
        _launch(c.device, (_lib or _load()).stream_cache8_write, (c._p8, *args), _checked_stream(stream, c.device))
    else:
        _launch(c.device, (_lib or _load()).stream_cache_write, (c._p, *args), _checked_stream(stream, c.device))


def cache_read(cache: PagedCache, cu: torch.Tensor, total: int, *, layer: int = 0, out: tuple[torch.Tensor, torch.Tensor] | None = None, stream=None):
    """Keys and values of a layer out of the pages, packed: rows ``cu[s] .. cu[s + 1]`` (int32 ``[n_slots + 1]``) are slot s's last tokens, as many
    of them. Returns k and v, ``[total, n_kv_heads, d]``, what :func:`prompt_attention` takes for prompts that come in pieces (or fills
    ``out``, a pair of them). Rows of no slot are left as they are, tokens without a page are zeros."""
    c = cache
    _checked(cu, torch.int32, (c.n_slots + 1,), "cu", c.device)
    if not 0 <= layer < c.n_layers:
        raise ValueError("no such layer")
    if not 0 <= total <= 0x7fffffff:
        raise ValueError("total must be 0 .. 2^31 - 1")
    if stream is not None:
        return _on_stream(stream, c.device, cache_read, c, cu, total, layer=layer, out=out)
    G, d = c.n_kv_heads, c.d
    if out is None:
        k, v = (torch.empty_strided((total, G, d), (G * d, d, 1), dtype=c.dtype, device=c.device) for _ in range(2))
    else:
        k, v = (_checked(x, c.dtype, (total, G, d), "out", c.device) for x in out)
    args = *c._pages(), cu.data_ptr(), total, c.page_table.data_ptr(), c.seq_len.data_ptr(), k.data_ptr(), v.data_ptr()
    if isinstance(c, PagedCache8):
        _launch(c.device, (_lib or _load()).stream_cache8_read, (c._p8, layer, *args), None)
    else:
        _launch(c.device, (_lib or _load()).stream_cache_read, (c._p, layer, *args), None)
    return k, v


def decode_attention(q: torch.Tensor, cache: PagedCache, *, layer: int = 0, scale: float = 0.0, window: int = 0, sinks: int = 0, want_lse: bool = False,
                     out: torch.Tensor | None = None, lse_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                     stream=None):
    """Attention of one new token of every slot, q ``[n_slots, H, d]``, over its cached tokens (with a ``window``, 0: none, over the last ``window``
    of them, its own among them, and the first ``sinks``). Returns the output
    ``[n_slots, H, d]``, with ``want_lse`` (or ``lse_out``) also the logarithms of the softmax sums, float32
    ``[n_slots, H]``. ``workspace``: uint8, at least :func:`stream_decode_workspace_bytes`, one per call that can overlap.
    Tokens whose page number is outside the cache are left out without an error here; the call's workspace has a record of them, which only
    one who gave it can look at (:func:`stream_read_stats` of it then raises, status ``STREAM_ERR_DEVICE_CHECK``)."""
    c, shape, strides = cache, q.shape, q.stride()
    if len(shape) != 3 or shape[0] != c.n_slots or shape[2] != c.d or q.dtype is not c.dtype or q.device != c.device:
        raise ValueError("q must be [n_slots, H, d] with the cache's dtype and device")
    if strides[2] != 1:
        raise ValueError("innermost stride must be 1")
    if not 0 <= layer < c.n_layers:
        raise ValueError("no such layer")
    if stream is not None:
        return _on_stream(stream, c.device, decode_attention, q, c, layer=layer, scale=scale, window=window, sinks=sinks, want_lse=want_lse, out=out,
                          lse_out=lse_out, workspace=workspace)
    if window or sinks:
        window, sinks = _window(window, sinks)
    n, H, d = shape
    if out is None:
        out = torch.empty_strided(shape, (H * d, d, 1), dtype=q.dtype, device=c.device)
    else:
        _checked(out, q.dtype, shape, "out", c.device)
    if lse_out is not None:
        _checked(lse_out, torch.float32, (n, H), "lse_out", c.device)
    elif want_lse:
        lse_out = torch.empty_strided((n, H), (H, 1), dtype=torch.float32, device=c.device)
    if workspace is None:
        need = c._decode_bytes.get(H) or stream_decode_workspace_bytes(c.struct, H)
        if need == 0:
            raise StreamError(STREAM_ERR_INVALID_ARG, stream_last_error())
        c._decode_bytes[H] = need
        workspace = torch.empty_strided((need,), (1,), dtype=torch.uint8, device=c.device)
    else:
        need = workspace.numel()
        if workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.device != c.device:
            raise ValueError("workspace must be a contiguous uint8 tensor on the cache's device")
    tail = (*c._pages(), c.page_table.data_ptr(), c.seq_len.data_ptr(), scale, out.data_ptr(), None if lse_out is None else lse_out.data_ptr(),
            workspace.data_ptr(), need)
    if isinstance(c, PagedCache8):
        _launch(c.device, (_lib or _load()).stream_decode_attention8, (c._p8, layer, H, window, sinks, q.data_ptr(), strides[0], strides[1], *tail), None)
    elif window:
        _launch(c.device, (_lib or _load()).stream_decode_window_attention, (c._p, layer, H, window, sinks, q.data_ptr(), strides[0], strides[1], *tail), None)
    else:
        _launch(c.device, (_lib or _load()).stream_decode_attention, (c._p, layer, H, q.data_ptr(), strides[0], strides[1], *tail), None)
    return out if lse_out is None else (out, lse_out)
