"""ctypes binding of libloma (declared in ``include/loma.h``).

Argument marshalling only: every function here has the name of the C entry
point it calls, takes torch tensors (device memory) or plain ints, pulls out
pointers, shapes and strides, and raises :class:`LomaError` on a negative
status.  No arithmetic of the method happens in Python, and there is no
fallback: if the library has not been built, loading fails with an error.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

LOMA_F32 = 0
LOMA_BF16 = 1
LOMA_FLAG_MEM_SEES_PRIOR_MEM = 1
LOMA_FLAG_NO_REP_ZONE = 2
LOMA_FLAG_FORCE_GENERIC = 1 << 8

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libloma.so")
_lib = None

_i, _i64, _f, _u, _p, _sz = (ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_uint, ctypes.c_void_p,
                             ctypes.c_size_t)

# name -> (restype, argtypes); mirrors include/loma.h
SIGNATURES = {
    "loma_layout_index": (_i, [_i, _i, _i, _i, _u, _p, _p, _p, _p, _p, _i, _p]),
    "loma_prefill_cache": (_i, [_p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i64, _i64, _i64, _i, _u, _p, _p]),
    "loma_generation_index": (_i, [_i, _i, _i, _p, _p, _p, _i, _p]),
    "loma_masked_attn_fwd": (_i, [_p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i64, _i64, _i64, _i, _f,
                                  _u, _p]),
    "loma_masked_attn_bwd": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i64, _i64, _i64, _i,
                                  _f, _u, _p, _sz, _p]),
    "loma_masked_attn_bwd_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _i, _u]),
    "loma_rope_apply": (_i, [_p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i64, _i64, _i64, _i, _f, _i, _u, _p]),
    "loma_masked_attn_plan_coverage": (_i, [_i, _i, _i, _i, _u, _p]),
    "loma_masked_attn_bwd_plan_coverage": (_i, [_i, _i, _i, _i, _u, _p]),
    "loma_prefill_attn": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _f, _u, _p]),
    "loma_prefill_attn_ragged": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _p, _i, _i, _f, _u, _p]),
    "loma_prefill_attn_paged": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _p, _i, _i, _f, _u, _p]),
    "loma_prefill_attn_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _f, _i, _f, _u, _p]),
    "loma_prefill_attn_ragged_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _p, _i, _p, _f, _i, _f, _u, _p]),
    "loma_prefill_attn_paged_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _p, _i, _p, _f, _i, _f,
                                          _u, _p]),
    "loma_prefill_attn_plan_coverage": (_i, [_i, _i, _p]),
    "loma_decode_attn": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _f, _u, _p, _sz, _p]),
    "loma_decode_attn_layers": (_i, [_i, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _f, _u, _p, _sz, _p]),
    "loma_compress_step_layers": (_i, [_i, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _f, _u, _p, _sz,
                                       _p]),
    "loma_decode_attn_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _f, _i, _f, _u, _p, _sz, _p]),
    "loma_compress_step_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _i, _f, _i, _f, _u, _p,
                                     _sz, _p]),
    "loma_decode_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "loma_decode_attn_paged": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _p, _i, _i, _f, _u, _p, _sz, _p]),
    "loma_decode_attn_ragged": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _p, _i, _i, _f, _u, _p, _sz, _p]),
    "loma_decode_attn_ragged_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _p, _i, _p, _f, _i, _f, _u, _p, _sz, _p]),
    "loma_decode_attn_paged_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _p, _i, _p, _f, _i, _f, _u, _p, _sz,
                                         _p]),
    "loma_compress_step_ragged_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _p, _i, _i, _i, _i, _p, _i, _f, _i, _f, _u, _p]),
    "loma_compress_step_paged_rope": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _p, _i, _i, _i, _i, _p, _i, _f, _i,
                                           _f, _u, _p]),
    "loma_decode_attn_static": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _f, _p]),
    "loma_decode_static_scratch_bytes": (_sz, []),
    "loma_compress_step": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _f, _u, _p, _sz,
                                _p]),
    "loma_compress_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _u]),
    "loma_compress_step_paged": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _p, _i, _i, _i, _i, _i, _f, _u, _p]),
    "loma_compress_step_ragged": (_i, [_p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _p, _i, _i, _i, _i, _i, _f, _u, _p]),
    "loma_paged_extend": (_i, [_i, _i, _i, _i, _i, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _i, _p]),
    "loma_qk_norm_rope_fwd": (_i, [_p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _p, _p, _i, _f, _f, _i, _u, _p]),
    "loma_qk_norm_rope_bwd": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _p, _p, _i, _f, _f,
                                   _i, _u, _p, _sz, _p]),
    "loma_qk_norm_rope_bwd_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _i, _i, _u]),
    "loma_qk_norm_rope_append": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _p, _p, _p, _i, _f, _f, _p]),
    "loma_decode_attn_shared": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _p, _i, _i, _f, _u, _p, _sz, _p]),
    "loma_decode_attn_shared_paged": (_i, [_p, _p, _p, _p, _p, _p, _p, _p, _p, _i, _i, _i, _i, _i, _i, _i, _i, _i, _p, _i, _i, _f, _u,
                                           _p, _sz, _p]),
    "loma_decode_shared_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "loma_device_status": (_i, [_p]),
    "loma_selftest_bounded_wait": (_i, [_p]),
    "loma_launch_count": (ctypes.c_uint64, []),
    "loma_fallback_count": (ctypes.c_uint64, []),
    "loma_status_string": (ctypes.c_char_p, [_i]),
    "loma_version": (_i, []),
}


class LomaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def library_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """Load libloma.so once.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2401_09486_b200.build` "
                "(there is no fallback path)")
        handle = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def status_string(status: int) -> str:
    return lib().loma_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise LomaError(status, where)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return LOMA_F32
    if t.dtype == torch.bfloat16:
        return LOMA_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    elif isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    return ctypes.c_void_p(int(stream))


def loma_version() -> int:
    return lib().loma_version()


def loma_launch_count() -> int:
    return int(lib().loma_launch_count())


def loma_fallback_count() -> int:
    """bf16 calls that ran on the CUDA-core kernels because the tensor-core path declined them."""
    return int(lib().loma_fallback_count())


def loma_selftest_bounded_wait(stream=None) -> None:
    _check(lib().loma_selftest_bounded_wait(_stream(stream)), "loma_selftest_bounded_wait")


def loma_device_status(stream=None) -> int:
    return lib().loma_device_status(_stream(stream))


def loma_layout_index(n_chunks: int, c: int, t: int, tail_read: int = 0, device="cpu", stream=None, flags: int = 0):
    """Returns int32 tensors (chunk, zone, offset, src_token, pos_id) on `device`."""
    tc = c * t
    S = n_chunks * ((tc + t) if (flags & LOMA_FLAG_NO_REP_ZONE) else (2 * tc + t)) + tail_read
    on_device = torch.device(device).type == "cuda"
    outs = [torch.empty(max(S, 0), dtype=torch.int32, device=device) for _ in range(5)]
    st = _stream(stream) if on_device else None
    rc = lib().loma_layout_index(n_chunks, c, t, tail_read, int(flags), *[_ptr(x) for x in outs], int(on_device), st)
    _check(rc, "loma_layout_index")
    return tuple(outs)


def loma_generation_index(n_tokens: int, c: int, t: int, device="cpu", stream=None):
    """Returns int32 tensors (slot, pos_id, compress_after) on `device`."""
    on_device = torch.device(device).type == "cuda"
    outs = [torch.empty(max(n_tokens, 0), dtype=torch.int32, device=device) for _ in range(3)]
    st = _stream(stream) if on_device else None
    rc = lib().loma_generation_index(n_tokens, c, t, *[_ptr(x) for x in outs], int(on_device), st)
    _check(rc, "loma_generation_index")
    return tuple(outs)


def loma_masked_attn_fwd(q, k, v, o, lse, n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0,
                         softmax_scale: float = 0.0, stream=None) -> None:
    """q, k, v, o: [B, H, S, D] device tensors with identical strides, D contiguous;
    lse: fp32 [B, H, S] contiguous or None."""
    B, H, S, D = q.shape
    for x in (k, v, o):
        if x.shape != q.shape or x.stride() != q.stride() or x.dtype != q.dtype:
            raise ValueError("q, k, v, o must share shape, strides and dtype")
    if q.stride(3) != 1:
        raise ValueError("head dimension must be contiguous")
    if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous fp32")
    rc = lib().loma_masked_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, H, D, n_chunks, c, t, c * t,
                                    tail_read, q.stride(0), q.stride(1), q.stride(2), _dtype_code(q),
                                    float(softmax_scale), int(flags), _stream(stream))
    _check(rc, "loma_masked_attn_fwd")


def loma_masked_attn_bwd_workspace_bytes(B: int, H: int, D: int, n_chunks: int, c: int, t: int, tail_read: int = 0,
                                         flags: int = 0) -> int:
    return int(lib().loma_masked_attn_bwd_workspace_bytes(B, H, D, n_chunks, c, t, tail_read, int(flags)))


def loma_masked_attn_bwd(q, k, v, o, d_o, lse, dq, dk, dv, n_chunks: int, c: int, t: int, tail_read: int = 0,
                         flags: int = 0, workspace=None, softmax_scale: float = 0.0, stream=None) -> None:
    """Gradients of loma_masked_attn_fwd.  q, k, v, o, d_o, dq, dk, dv: [B, H, S, D] device tensors with
    identical strides; lse: the forward's fp32 [B, H, S]; workspace: a device byte buffer of at least
    loma_masked_attn_bwd_workspace_bytes(...) bytes."""
    B, H, S, D = q.shape
    for x in (k, v, o, d_o, dq, dk, dv):
        if x.shape != q.shape or x.stride() != q.stride() or x.dtype != q.dtype:
            raise ValueError("all tensors must share shape, strides and dtype")
    if q.stride(3) != 1:
        raise ValueError("head dimension must be contiguous")
    if lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be contiguous fp32")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_masked_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), _ptr(dq), _ptr(dk),
                                    _ptr(dv), B, H, D, n_chunks, c, t, c * t, tail_read, q.stride(0), q.stride(1),
                                    q.stride(2), _dtype_code(q), float(softmax_scale), int(flags), _ptr(workspace),
                                    ws_bytes, _stream(stream))
    _check(rc, "loma_masked_attn_bwd")


def loma_masked_attn_plan_coverage(n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0) -> torch.Tensor:
    """Host replay of the tensor-core kernel's tile plan: uint8 [S, S] visit counts."""
    S = n_chunks * ((c * t + t) if (flags & LOMA_FLAG_NO_REP_ZONE) else (2 * c * t + t)) + tail_read
    counts = torch.empty((S, S), dtype=torch.uint8)
    rc = lib().loma_masked_attn_plan_coverage(n_chunks, c, t, tail_read, int(flags), _ptr(counts))
    _check(rc, "loma_masked_attn_plan_coverage")
    return counts


def loma_prefill_attn(q, k_new, v_new, k_cache, v_cache, o, lse, cache_len: int, flags: int = 0,
                      softmax_scale: float = 0.0, stream=None) -> None:
    """q, k_new, v_new, o: [B, H, l, D] contiguous; caches [B, H, cap, D] contiguous; appends then attends."""
    B, H, l, D = q.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o):
        if x is not None and not x.is_contiguous():
            raise ValueError("loma_prefill_attn takes contiguous tensors")
    rc = lib().loma_prefill_attn(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse),
                                 B, H, D, l, k_cache.shape[2], int(cache_len), _dtype_code(q), float(softmax_scale),
                                 int(flags), _stream(stream))
    _check(rc, "loma_prefill_attn")


def loma_prefill_attn_ragged(q, k_new, v_new, k_cache, v_cache, o, lse, cache_lens, max_cache_len: int, flags: int = 0,
                             softmax_scale: float = 0.0, stream=None) -> None:
    """loma_prefill_attn with one cache length per sequence (cache_lens: int32 [B] on the device)."""
    B, H, l, D = q.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o):
        if x is not None and not x.is_contiguous():
            raise ValueError("loma_prefill_attn_ragged takes contiguous tensors")
    if cache_lens.dtype != torch.int32 or cache_lens.numel() != B or not cache_lens.is_contiguous():
        raise ValueError("cache_lens must be a contiguous int32 tensor of B entries")
    rc = lib().loma_prefill_attn_ragged(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse),
                                        B, H, D, l, k_cache.shape[2], _ptr(cache_lens), int(max_cache_len), _dtype_code(q),
                                        float(softmax_scale), int(flags), _stream(stream))
    _check(rc, "loma_prefill_attn_ragged")


def loma_prefill_attn_paged(q, k_new, v_new, k_pool, v_pool, block_table, o, lse, cache_lens, max_cache_len: int,
                            flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """loma_prefill_attn over a paged cache: pools [n_pages, H, page_size, D], block_table int32 [B, max_pages]."""
    B, H, l, D = q.shape
    for x in (q, k_new, v_new, k_pool, v_pool, o, block_table):
        if x is not None and not x.is_contiguous():
            raise ValueError("loma_prefill_attn_paged takes contiguous tensors")
    if cache_lens.dtype != torch.int32 or cache_lens.numel() != B or block_table.dtype != torch.int32:
        raise ValueError("cache_lens and block_table must be int32")
    n_pages, _, page_size, _ = k_pool.shape
    rc = lib().loma_prefill_attn_paged(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                       _ptr(o), _ptr(lse), B, H, D, l, page_size, block_table.shape[1], n_pages,
                                       _ptr(cache_lens), int(max_cache_len), _dtype_code(q), float(softmax_scale),
                                       int(flags), _stream(stream))
    _check(rc, "loma_prefill_attn_paged")


def loma_prefill_attn_rope(q, k_new, v_new, k_cache, v_cache, o, lse, cache_len: int, pos0: int, flags: int = 0,
                           softmax_scale: float = 0.0, theta_base: float = 0.0, stream=None) -> None:
    """loma_prefill_attn with q and k_new rotated at the ids pos0 .. pos0 + l - 1 on the way in."""
    B, H, l, D = q.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o):
        if x is not None and not x.is_contiguous():
            raise ValueError("loma_prefill_attn_rope takes contiguous tensors")
    rc = lib().loma_prefill_attn_rope(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse),
                                      B, H, D, l, k_cache.shape[2], int(cache_len), int(pos0), float(theta_base),
                                      _dtype_code(q), float(softmax_scale), int(flags), _stream(stream))
    _check(rc, "loma_prefill_attn_rope")


def loma_prefill_attn_ragged_rope(q, k_new, v_new, k_cache, v_cache, o, lse, cache_lens, max_cache_len: int, positions,
                                  flags: int = 0, softmax_scale: float = 0.0, theta_base: float = 0.0, stream=None) -> None:
    """loma_prefill_attn_ragged with the rotation fused in; positions: int32 [B], id of every sequence's first new token."""
    B, H, l, D = q.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o):
        if x is not None and not x.is_contiguous():
            raise ValueError("loma_prefill_attn_ragged_rope takes contiguous tensors")
    _check_positions(positions, B, "positions")
    rc = lib().loma_prefill_attn_ragged_rope(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o),
                                             _ptr(lse), B, H, D, l, k_cache.shape[2], _ptr(cache_lens), int(max_cache_len),
                                             _ptr(positions), float(theta_base), _dtype_code(q), float(softmax_scale),
                                             int(flags), _stream(stream))
    _check(rc, "loma_prefill_attn_ragged_rope")


def loma_prefill_attn_paged_rope(q, k_new, v_new, k_pool, v_pool, block_table, o, lse, cache_lens, max_cache_len: int,
                                 positions, flags: int = 0, softmax_scale: float = 0.0, theta_base: float = 0.0,
                                 stream=None) -> None:
    """loma_prefill_attn_paged with the rotation fused in."""
    B, H, l, D = q.shape
    _check_positions(positions, B, "positions")
    n_pages, _, page_size, _ = k_pool.shape
    rc = lib().loma_prefill_attn_paged_rope(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                            _ptr(o), _ptr(lse), B, H, D, l, page_size, block_table.shape[1], n_pages,
                                            _ptr(cache_lens), int(max_cache_len), _ptr(positions), float(theta_base),
                                            _dtype_code(q), float(softmax_scale), int(flags), _stream(stream))
    _check(rc, "loma_prefill_attn_paged_rope")


def loma_prefill_attn_plan_coverage(l: int, cache_len: int) -> torch.Tensor:
    """Host replay of the tensor-core kernel's tile plan for loma_prefill_attn: uint8 [l, cache_len + l] visit counts."""
    counts = torch.empty((l, cache_len + l), dtype=torch.uint8)
    rc = lib().loma_prefill_attn_plan_coverage(int(l), int(cache_len), _ptr(counts))
    _check(rc, "loma_prefill_attn_plan_coverage")
    return counts


def loma_masked_attn_bwd_plan_coverage(n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0) -> torch.Tensor:
    """Host replay of the key-tile side of the plan (the backward's dK/dV pass): uint8 [S, S] visit counts."""
    S = n_chunks * ((c * t + t) if (flags & LOMA_FLAG_NO_REP_ZONE) else (2 * c * t + t)) + tail_read
    counts = torch.empty((S, S), dtype=torch.uint8)
    rc = lib().loma_masked_attn_bwd_plan_coverage(n_chunks, c, t, tail_read, int(flags), _ptr(counts))
    _check(rc, "loma_masked_attn_bwd_plan_coverage")
    return counts


LOMA_ROPE_INVERSE = 2


def loma_rope_apply(q, k, n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0, theta_base: float = 0.0,
                    position_type: int = 0, stream=None) -> None:
    """Rotates q and k ([B, H, S, D] device tensors with identical strides; either may be None) in place at
    the layout's position ids.  position_type 0: Eq. 14; 1: the generator's contiguous memory ids."""
    ref = q if q is not None else k
    B, H, S, D = ref.shape
    if q is not None and k is not None and (k.shape != q.shape or k.stride() != q.stride() or k.dtype != q.dtype):
        raise ValueError("q and k must share shape, strides and dtype")
    if ref.stride(3) != 1:
        raise ValueError("head dimension must be contiguous")
    rc = lib().loma_rope_apply(_ptr(q), _ptr(k), B, H, D, n_chunks, c, t, c * t, tail_read, ref.stride(0), ref.stride(1),
                               ref.stride(2), _dtype_code(ref), float(theta_base), int(position_type), int(flags),
                               _stream(stream))
    _check(rc, "loma_rope_apply")


def loma_prefill_cache(k, v, k_cache, v_cache, n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0,
                       stream=None) -> int:
    """Gathers the memory-zone rows and the reading tail of laid-out k, v [B, H, S, D] into the caches
    [B, H, cap, D]; returns the new cache length."""
    B, H, S, D = k.shape
    if v.shape != k.shape or v.stride() != k.stride() or k.stride(3) != 1:
        raise ValueError("k and v must share shape and strides, head dimension contiguous")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("caches must be contiguous")
    n = ctypes.c_int(0)
    rc = lib().loma_prefill_cache(_ptr(k), _ptr(v), _ptr(k_cache), _ptr(v_cache), B, H, D, k_cache.shape[2], n_chunks, c,
                                  t, c * t, tail_read, k.stride(0), k.stride(1), k.stride(2), _dtype_code(k), int(flags),
                                  ctypes.byref(n), _stream(stream))
    _check(rc, "loma_prefill_cache")
    return n.value


def loma_decode_workspace_bytes(B: int, H: int, D: int, cache_len: int) -> int:
    return int(lib().loma_decode_workspace_bytes(B, H, D, cache_len))


def loma_decode_attn(q, k_new, v_new, k_cache, v_cache, o, lse, cache_len: int, workspace=None, flags: int = 0,
                     softmax_scale: float = 0.0, stream=None) -> None:
    """q, k_new, v_new, o: [B, H, 1, D]; caches [B, H, cap, D]; all contiguous."""
    B, H, cap, D = k_cache.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o):
        if x is not None and not x.is_contiguous():
            raise ValueError("decode tensors must be contiguous")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_decode_attn(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o),
                                _ptr(lse), B, H, D, cap, cache_len, _dtype_code(q), float(softmax_scale),
                                int(flags), _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_decode_attn")


def _ptr_array(tensors):
    """[host] array of device pointers, one per layer (None stays NULL)."""
    if tensors is None:
        return None
    arr = (ctypes.c_void_p * len(tensors))()
    for i, x in enumerate(tensors):
        arr[i] = None if x is None else x.data_ptr()
    return arr


def loma_decode_attn_layers(q, k_new, v_new, k_cache, v_cache, o, lse, cache_len: int, workspace=None, flags: int = 0,
                            softmax_scale: float = 0.0, stream=None) -> None:
    """Lists of per-layer tensors (shapes of loma_decode_attn); k_new, v_new, lse may be None."""
    n = len(q)
    B, H, cap, D = k_cache[0].shape
    for group in (q, k_new, v_new, k_cache, v_cache, o):
        for x in (group or []):
            if x is not None and not x.is_contiguous():
                raise ValueError("decode tensors must be contiguous")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    arrays = [_ptr_array(x) for x in (q, k_new, v_new, k_cache, v_cache, o, lse)]
    rc = lib().loma_decode_attn_layers(n, *arrays, B, H, D, cap, cache_len, _dtype_code(q[0]), float(softmax_scale), int(flags),
                                       _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_decode_attn_layers")


def loma_compress_step_layers(q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, lse, mem_len: int, c: int, t: int, workspace=None,
                              flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """Lists of per-layer tensors (shapes of loma_compress_step); lse may be None."""
    n = len(q_mem)
    B, H, cap, D = k_cache[0].shape
    for group in (q_mem, k_mem, v_mem, k_cache, v_cache, o_mem):
        for x in group:
            if not x.is_contiguous():
                raise ValueError("compress tensors must be contiguous")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    arrays = [_ptr_array(x) for x in (q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, lse)]
    rc = lib().loma_compress_step_layers(n, *arrays, B, H, D, cap, mem_len, c, t, c * t, _dtype_code(q_mem[0]),
                                         float(softmax_scale), int(flags), _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_compress_step_layers")


def loma_decode_attn_rope(q, k_new, v_new, k_cache, v_cache, o, lse, cache_len: int, pos: int, workspace=None,
                          flags: int = 0, softmax_scale: float = 0.0, theta_base: float = 0.0, stream=None) -> None:
    """loma_decode_attn with q and k_new rotated inside the step by the position id `pos`."""
    B, H, cap, D = k_cache.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o):
        if x is not None and not x.is_contiguous():
            raise ValueError("decode tensors must be contiguous")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_decode_attn_rope(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o),
                                     _ptr(lse), B, H, D, cap, cache_len, int(pos), float(theta_base), _dtype_code(q),
                                     float(softmax_scale), int(flags), _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_decode_attn_rope")


def loma_compress_step_rope(q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, lse, mem_len: int, c: int, t: int, pos0: int,
                            pos_stride: int, workspace=None, flags: int = 0, softmax_scale: float = 0.0,
                            theta_base: float = 0.0, stream=None) -> None:
    """loma_compress_step with memory row j's query and key rotated inside the step by the id pos0 + j * pos_stride."""
    B, H, cap, D = k_cache.shape
    for x in (q_mem, k_mem, v_mem, k_cache, v_cache, o_mem):
        if not x.is_contiguous():
            raise ValueError("compress tensors must be contiguous")
    if q_mem.shape[2] != t:
        raise ValueError("q_mem must have t rows")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_compress_step_rope(_ptr(q_mem), _ptr(k_mem), _ptr(v_mem), _ptr(k_cache), _ptr(v_cache), _ptr(o_mem),
                                       _ptr(lse), B, H, D, cap, mem_len, c, t, c * t, int(pos0), int(pos_stride),
                                       float(theta_base), _dtype_code(q_mem), float(softmax_scale), int(flags),
                                       _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_compress_step_rope")


def loma_decode_attn_ragged(q, k_new, v_new, k_cache, v_cache, o, lse, cache_lens, max_cache_len: int, workspace=None,
                            flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """loma_decode_attn with one cache length per sequence: cache_lens is a device int32 [B] tensor,
    max_cache_len a host-side upper bound of its entries."""
    B, H, cap, D = k_cache.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o, cache_lens):
        if x is not None and not x.is_contiguous():
            raise ValueError("decode tensors must be contiguous")
    if cache_lens.dtype != torch.int32 or cache_lens.numel() != B:
        raise ValueError("cache_lens must be int32 [B]")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_decode_attn_ragged(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o),
                                       _ptr(lse), B, H, D, cap, _ptr(cache_lens), int(max_cache_len), _dtype_code(q),
                                       float(softmax_scale), int(flags), _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_decode_attn_ragged")


def loma_decode_attn_paged(q, k_new, v_new, k_pool, v_pool, block_table, o, lse, cache_lens, max_cache_len: int,
                           workspace=None, flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """Ragged decode over a paged cache.  k_pool, v_pool: [n_pages, H, page_size, D]; block_table: device int32
    [B, max_pages]; cache_lens: device int32 [B]; q, k_new, v_new, o: [B, H, 1, D]."""
    n_pages, H, page_size, D = k_pool.shape
    B, max_pages = block_table.shape
    for x in (q, k_new, v_new, k_pool, v_pool, o, block_table, cache_lens):
        if x is not None and not x.is_contiguous():
            raise ValueError("decode tensors must be contiguous")
    if block_table.dtype != torch.int32 or cache_lens.dtype != torch.int32 or cache_lens.numel() != B:
        raise ValueError("block_table must be int32 [B, max_pages] and cache_lens int32 [B]")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_decode_attn_paged(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                      _ptr(o), _ptr(lse), B, H, D, page_size, max_pages, n_pages, _ptr(cache_lens),
                                      int(max_cache_len), _dtype_code(q), float(softmax_scale), int(flags),
                                      _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_decode_attn_paged")


def _check_positions(positions, B, what):
    if positions.dtype != torch.int32 or positions.numel() != B or not positions.is_contiguous():
        raise ValueError(f"{what} must be a contiguous int32 [B] tensor")


def loma_decode_attn_ragged_rope(q, k_new, v_new, k_cache, v_cache, o, lse, cache_lens, max_cache_len: int, positions,
                                 workspace=None, flags: int = 0, softmax_scale: float = 0.0, theta_base: float = 0.0,
                                 stream=None) -> None:
    """loma_decode_attn_ragged with q and k_new of sequence b rotated inside the step by positions[b] (device int32 [B])."""
    B, H, cap, D = k_cache.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o, cache_lens):
        if x is not None and not x.is_contiguous():
            raise ValueError("decode tensors must be contiguous")
    if cache_lens.dtype != torch.int32 or cache_lens.numel() != B:
        raise ValueError("cache_lens must be int32 [B]")
    _check_positions(positions, B, "positions")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_decode_attn_ragged_rope(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse),
                                            B, H, D, cap, _ptr(cache_lens), int(max_cache_len), _ptr(positions),
                                            float(theta_base), _dtype_code(q), float(softmax_scale), int(flags),
                                            _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_decode_attn_ragged_rope")


def loma_decode_attn_paged_rope(q, k_new, v_new, k_pool, v_pool, block_table, o, lse, cache_lens, max_cache_len: int, positions,
                                workspace=None, flags: int = 0, softmax_scale: float = 0.0, theta_base: float = 0.0,
                                stream=None) -> None:
    """loma_decode_attn_paged with the rotation fused in (positions: device int32 [B])."""
    n_pages, H, page_size, D = k_pool.shape
    B, max_pages = block_table.shape
    for x in (q, k_new, v_new, k_pool, v_pool, o, block_table, cache_lens):
        if x is not None and not x.is_contiguous():
            raise ValueError("decode tensors must be contiguous")
    if block_table.dtype != torch.int32 or cache_lens.dtype != torch.int32 or cache_lens.numel() != B:
        raise ValueError("block_table must be int32 [B, max_pages] and cache_lens int32 [B]")
    _check_positions(positions, B, "positions")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_decode_attn_paged_rope(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                           _ptr(o), _ptr(lse), B, H, D, page_size, max_pages, n_pages, _ptr(cache_lens),
                                           int(max_cache_len), _ptr(positions), float(theta_base), _dtype_code(q),
                                           float(softmax_scale), int(flags), _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_decode_attn_paged_rope")


def loma_compress_step_ragged_rope(q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, lse, mem_lens, max_mem_len: int, c: int, t: int,
                                   pos0s, pos_stride: int, flags: int = 0, softmax_scale: float = 0.0, theta_base: float = 0.0,
                                   stream=None) -> None:
    """loma_compress_step_ragged with memory row j of sequence b rotated by pos0s[b] + j * pos_stride inside the step."""
    B, H, cap, D = k_cache.shape
    for x in (q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, mem_lens):
        if not x.is_contiguous():
            raise ValueError("compress tensors must be contiguous")
    if mem_lens.dtype != torch.int32 or mem_lens.numel() != B:
        raise ValueError("mem_lens must be int32 [B]")
    _check_positions(pos0s, B, "pos0s")
    rc = lib().loma_compress_step_ragged_rope(_ptr(q_mem), _ptr(k_mem), _ptr(v_mem), _ptr(k_cache), _ptr(v_cache), _ptr(o_mem),
                                              _ptr(lse), B, H, D, cap, _ptr(mem_lens), int(max_mem_len), c, t, c * t,
                                              _ptr(pos0s), int(pos_stride), float(theta_base), _dtype_code(q_mem),
                                              float(softmax_scale), int(flags), _stream(stream))
    _check(rc, "loma_compress_step_ragged_rope")


def loma_compress_step_paged_rope(q_mem, k_mem, v_mem, k_pool, v_pool, block_table, o_mem, lse, mem_lens, max_mem_len: int,
                                  c: int, t: int, pos0s, pos_stride: int, flags: int = 0, softmax_scale: float = 0.0,
                                  theta_base: float = 0.0, stream=None) -> None:
    """loma_compress_step_paged with the rotation fused in (pos0s: device int32 [B])."""
    n_pages, H, page_size, D = k_pool.shape
    B, max_pages = block_table.shape
    for x in (q_mem, k_mem, v_mem, k_pool, v_pool, o_mem, mem_lens, block_table):
        if not x.is_contiguous():
            raise ValueError("compress tensors must be contiguous")
    if block_table.dtype != torch.int32 or mem_lens.dtype != torch.int32 or mem_lens.numel() != B:
        raise ValueError("block_table must be int32 [B, max_pages] and mem_lens int32 [B]")
    _check_positions(pos0s, B, "pos0s")
    rc = lib().loma_compress_step_paged_rope(_ptr(q_mem), _ptr(k_mem), _ptr(v_mem), _ptr(k_pool), _ptr(v_pool),
                                             _ptr(block_table), _ptr(o_mem), _ptr(lse), B, H, D, page_size, max_pages, n_pages,
                                             _ptr(mem_lens), int(max_mem_len), c, t, c * t, _ptr(pos0s), int(pos_stride),
                                             float(theta_base), _dtype_code(q_mem), float(softmax_scale), int(flags),
                                             _stream(stream))
    _check(rc, "loma_compress_step_paged_rope")


def loma_decode_static_scratch_bytes() -> int:
    return int(lib().loma_decode_static_scratch_bytes())


def loma_decode_attn_static(q, k_new, v_new, k_cache, v_cache, o, lse, cache_len: int, softmax_scale: float = 0.0,
                            stream=None) -> None:
    """loma_decode_attn without a workspace argument: the split partials go to
    the library's built-in 8 MiB array, so the call needs no device memory beyond
    the tensors passed in.  Same tensor conventions as loma_decode_attn (bf16)."""
    B, H, cap, D = k_cache.shape
    for x in (q, k_new, v_new, k_cache, v_cache, o):
        if x is not None and not x.is_contiguous():
            raise ValueError("decode tensors must be contiguous")
    rc = lib().loma_decode_attn_static(_ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(o),
                                       _ptr(lse), B, H, D, cap, cache_len, _dtype_code(q), float(softmax_scale),
                                       _stream(stream))
    _check(rc, "loma_decode_attn_static")


def loma_compress_step_ragged(q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, lse, mem_lens, max_mem_len: int, c: int, t: int,
                              flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """loma_compress_step with one count of memory entries per sequence (device int32 [B]; negative = the
    sequence does not compress in this call)."""
    B, H, cap, D = k_cache.shape
    for x in (q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, mem_lens):
        if not x.is_contiguous():
            raise ValueError("compress tensors must be contiguous")
    if mem_lens.dtype != torch.int32 or mem_lens.numel() != B:
        raise ValueError("mem_lens must be int32 [B]")
    rc = lib().loma_compress_step_ragged(_ptr(q_mem), _ptr(k_mem), _ptr(v_mem), _ptr(k_cache), _ptr(v_cache), _ptr(o_mem),
                                         _ptr(lse), B, H, D, cap, _ptr(mem_lens), int(max_mem_len), c, t, c * t,
                                         _dtype_code(q_mem), float(softmax_scale), int(flags), _stream(stream))
    _check(rc, "loma_compress_step_ragged")


def loma_compress_step_paged(q_mem, k_mem, v_mem, k_pool, v_pool, block_table, o_mem, lse, mem_lens, max_mem_len: int,
                             c: int, t: int, flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """Ragged compress over a paged cache (pools [n_pages, H, page_size, D], block_table int32 [B, max_pages])."""
    n_pages, H, page_size, D = k_pool.shape
    B, max_pages = block_table.shape
    for x in (q_mem, k_mem, v_mem, k_pool, v_pool, o_mem, mem_lens, block_table):
        if not x.is_contiguous():
            raise ValueError("compress tensors must be contiguous")
    if block_table.dtype != torch.int32 or mem_lens.dtype != torch.int32 or mem_lens.numel() != B:
        raise ValueError("block_table must be int32 [B, max_pages] and mem_lens int32 [B]")
    rc = lib().loma_compress_step_paged(_ptr(q_mem), _ptr(k_mem), _ptr(v_mem), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                        _ptr(o_mem), _ptr(lse), B, H, D, page_size, max_pages, n_pages, _ptr(mem_lens),
                                        int(max_mem_len), c, t, c * t, _dtype_code(q_mem), float(softmax_scale), int(flags),
                                        _stream(stream))
    _check(rc, "loma_compress_step_paged")


def loma_compress_workspace_bytes(B: int, H: int, D: int, t: int, mem_len: int, flags: int = 0) -> int:
    return int(lib().loma_compress_workspace_bytes(B, H, D, t, mem_len, int(flags)))


def loma_compress_step(q_mem, k_mem, v_mem, k_cache, v_cache, o_mem, lse, mem_len: int, c: int, t: int,
                       workspace=None, flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """q_mem, k_mem, v_mem, o_mem: [B, H, t, D]; caches [B, H, cap, D]; all contiguous."""
    B, H, cap, D = k_cache.shape
    for x in (q_mem, k_mem, v_mem, k_cache, v_cache, o_mem):
        if not x.is_contiguous():
            raise ValueError("compress tensors must be contiguous")
    if q_mem.shape[2] != t:
        raise ValueError("q_mem must have t rows")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().loma_compress_step(_ptr(q_mem), _ptr(k_mem), _ptr(v_mem), _ptr(k_cache), _ptr(v_cache),
                                  _ptr(o_mem), _ptr(lse), B, H, D, cap, mem_len, c, t, c * t, _dtype_code(q_mem),
                                  float(softmax_scale), int(flags), _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "loma_compress_step")


# ---- one serving step: page tables, norm + rotation into the pages, attention over a shared prefix -----------------------

# Small calls are bound by the host, and a check of a tensor costs more than a kernel argument: the checks below ask each
# tensor only what they need (dtype objects are singletons, get_device() is -1 on the host), and name the culprit only
# once something is wrong.

def _addr(x) -> Optional[int]:
    return None if x is None else x.data_ptr()


def _on_current(where: str, dev: int) -> None:
    """A pointer of another device than the current one would reach the wrong GPU's kernel."""
    if dev < 0:
        raise ValueError(f"{where}: tensors must be on a CUDA device")
    if dev != torch.cuda.current_device():
        raise ValueError(f"{where}: tensors on cuda:{dev}, but the current device is cuda:{torch.cuda.current_device()}")


def _raw_stream(stream, dev: int) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


def _int32(where: str, dev: int, name: str, x, numel: int) -> None:
    """x is None, or contiguous int32 on device `dev` with `numel` entries (any number if negative)."""
    if x is not None and (x.dtype is not torch.int32 or x.get_device() != dev or not x.is_contiguous()
                          or (numel >= 0 and x.numel() != numel)):
        raise ValueError(f"{where}: {name} must be a contiguous int32 tensor on the call's device"
                         + (f" with {numel} entries" if numel >= 0 else ""))


def _expect(where: str, dev: int, name: str, x, shape, dtype) -> None:
    """x is None, or a contiguous tensor on device `dev` of this shape and dtype."""
    if x is not None and (x.dtype is not dtype or x.get_device() != dev or x.shape != shape or not x.is_contiguous()):
        raise ValueError(f"{where}: {name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the call's device")


def _scratch(where: str, dev: int, x) -> int:
    """Bytes of a workspace tensor."""
    if x is None:
        return 0
    if x.get_device() != dev or not x.is_contiguous():
        raise ValueError(f"{where}: workspace must be a contiguous tensor on the call's device")
    return x.numel() * x.element_size()


def _strides(x, axes):
    """[host] int64 array; an axis of one element has no stride of its own (torch reports any number there)."""
    shape, stride = x.shape, x.stride()
    return (ctypes.c_int64 * len(axes))(*[stride[a] if shape[a] > 1 else 0 for a in axes])


def loma_paged_extend(cache_lens, new_lens, held, pos0, free_pages, taken, block_table, page_size: int, row_start, page_start,
                      held_out, slots, row_seq, row_pos, stream=None) -> None:
    """Block table and slot maps from request lengths (see include/loma.h).  int32 tensors, all on the device or all on the
    host: cache_lens, new_lens, held, pos0 [B] (all but cache_lens may be None), free_pages, taken [1] or None, block_table
    [B, max_pages] (in/out); outputs row_start, page_start [B+1], held_out [B] (may be `held`), slots, row_seq, row_pos [rows]."""
    w = "loma_paged_extend"
    B, dev, rows = cache_lens.numel(), cache_lens.get_device(), slots.numel()
    _int32(w, dev, "cache_lens", cache_lens, B)
    _int32(w, dev, "new_lens", new_lens, B)
    _int32(w, dev, "held", held, B)
    _int32(w, dev, "pos0", pos0, B)
    _int32(w, dev, "free_pages", free_pages, -1)
    _int32(w, dev, "taken", taken, 1)
    _int32(w, dev, "block_table", block_table, -1)
    _int32(w, dev, "row_start", row_start, B + 1)
    _int32(w, dev, "page_start", page_start, B + 1)
    _int32(w, dev, "held_out", held_out, B)
    _int32(w, dev, "slots", slots, rows)
    _int32(w, dev, "row_seq", row_seq, rows)
    _int32(w, dev, "row_pos", row_pos, rows)
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError(f"{w}: block_table must be [B, max_pages]")
    if dev >= 0:
        _on_current(w, dev)
    rc = lib().loma_paged_extend(B, page_size, block_table.shape[1], rows, 0 if free_pages is None else free_pages.numel(),
                                 cache_lens.data_ptr(), _addr(new_lens), _addr(held), _addr(pos0), _addr(free_pages), _addr(taken),
                                 block_table.data_ptr(), row_start.data_ptr(), page_start.data_ptr(), held_out.data_ptr(),
                                 slots.data_ptr(), row_seq.data_ptr(), row_pos.data_ptr(), int(dev >= 0),
                                 _raw_stream(stream, dev) if dev >= 0 else None)
    _check(rc, w)


def _norm_args(where, q, k, wq, wk, pairs, gains, n_chunks, c, t, tail_read, flags):
    """Checks of the training-layout norm; returns (device, B, Hq, Hk, D, dtype code, q strides, k strides)."""
    if q.dim() != 4 or k.dim() != 4 or q.shape[0] != k.shape[0] or q.shape[2:] != k.shape[2:] or q.dtype is not k.dtype:
        raise ValueError(f"{where}: q [B, Hq, S, D] and k [B, Hk, S, D] must share B, S, D and dtype")
    B, Hq, S, D = q.shape
    Hk, dev, dtype = k.shape[1], q.get_device(), q.dtype
    if q.stride(3) != 1 or k.stride(3) != 1:
        raise ValueError(f"{where}: head dimension must be contiguous")
    if k.get_device() != dev:
        raise ValueError(f"{where}: q and k on different devices")
    for ref, x in pairs:
        if x.dtype is not dtype or x.get_device() != dev or x.shape != ref.shape or (
                x.stride() != ref.stride() and any(n > 1 and a != b for n, a, b in zip(x.shape, x.stride(), ref.stride()))):
            raise ValueError(f"{where}: every tensor that goes with q or k must have its shape, strides, dtype and device")
    for name, x in gains:
        _expect(where, dev, name, x, (D,), dtype)
    rows = n_chunks * ((c * t + t) if (flags & LOMA_FLAG_NO_REP_ZONE) else (2 * c * t + t)) + tail_read
    if S != rows:
        raise ValueError(f"{where}: the layout has {rows} rows, the tensors {S}")
    _on_current(where, dev)
    return dev, B, Hq, Hk, D, _dtype_code(q), _strides(q, (0, 1, 2)), _strides(k, (0, 1, 2))


def loma_qk_norm_rope_fwd(q, k, wq, wk, q_out, k_out, n_chunks: int, c: int, t: int, tail_read: int = 0, flags: int = 0,
                          eps: float = 0.0, theta_base: float = 0.0, position_type: int = 0, stream=None) -> None:
    """RMS norm of every head of q [B, Hq, S, D] and k [B, Hk, S, D] (gains wq, wk [D] or None) and the rotary embedding at the
    layout's position ids, in one pass.  q_out, k_out: shape and strides of q and k; q and k themselves are allowed."""
    w = "loma_qk_norm_rope_fwd"
    dev, B, Hq, Hk, D, dt, qs, ks = _norm_args(w, q, k, wq, wk, ((q, q_out), (k, k_out)), (("wq", wq), ("wk", wk)), n_chunks, c, t,
                                               tail_read, flags)
    rc = lib().loma_qk_norm_rope_fwd(q.data_ptr(), k.data_ptr(), _addr(wq), _addr(wk), q_out.data_ptr(), k_out.data_ptr(), B, Hq, Hk, D,
                                     n_chunks, c, t, c * t, tail_read, qs, ks, dt, eps, theta_base, position_type, flags,
                                     _raw_stream(stream, dev))
    _check(rc, w)


def loma_qk_norm_rope_bwd_workspace_bytes(B: int, Hq: int, Hk: int, D: int, n_chunks: int, c: int, t: int, tail_read: int = 0,
                                          flags: int = 0) -> int:
    return int(lib().loma_qk_norm_rope_bwd_workspace_bytes(B, Hq, Hk, D, n_chunks, c, t, tail_read, int(flags)))


def loma_qk_norm_rope_bwd(q, k, wq, wk, d_q_out, d_k_out, dq, dk, dwq, dwk, n_chunks: int, c: int, t: int, tail_read: int = 0,
                          flags: int = 0, workspace=None, eps: float = 0.0, theta_base: float = 0.0, position_type: int = 0,
                          stream=None) -> None:
    """Gradients of loma_qk_norm_rope_fwd at q, k, wq, wk.  d_q_out, dq have q's shape and strides, d_k_out, dk those of k;
    dwq, dwk [D] or None; workspace: a device byte buffer of loma_qk_norm_rope_bwd_workspace_bytes(...) bytes."""
    w = "loma_qk_norm_rope_bwd"
    dev, B, Hq, Hk, D, dt, qs, ks = _norm_args(w, q, k, wq, wk, ((q, d_q_out), (q, dq), (k, d_k_out), (k, dk)),
                                               (("wq", wq), ("wk", wk), ("dwq", dwq), ("dwk", dwk)), n_chunks, c, t, tail_read, flags)
    ws_bytes = _scratch(w, dev, workspace)
    rc = lib().loma_qk_norm_rope_bwd(q.data_ptr(), k.data_ptr(), _addr(wq), _addr(wk), d_q_out.data_ptr(), d_k_out.data_ptr(),
                                     dq.data_ptr(), dk.data_ptr(), _addr(dwq), _addr(dwk), B, Hq, Hk, D, n_chunks, c, t, c * t, tail_read,
                                     qs, ks, dt, eps, theta_base, position_type, flags, _addr(workspace), ws_bytes,
                                     _raw_stream(stream, dev))
    _check(rc, w)


def loma_qk_norm_rope_append(q, k_new, v_new, wq, wk, q_out, k_pool, v_pool, slots, positions, eps: float = 0.0,
                             theta_base: float = 0.0, stream=None) -> None:
    """Norm and rotation of T packed new tokens: q [T, Hq, D] into q_out (contiguous), k_new [T, Hk, D] and, copied, v_new into
    the pools [n_pages, Hk, page_size, D] at slots[r] = page * page_size + row (a slot outside the pool: not stored).
    slots, positions: int32 [T].  q, k_new, v_new may be views of one projection's output."""
    w = "loma_qk_norm_rope_append"
    if q.dim() != 3 or k_new.dim() != 3 or k_pool.dim() != 4:
        raise ValueError(f"{w}: q [T, Hq, D], k_new, v_new [T, Hk, D], pools [n_pages, Hk, page_size, D]")
    T, Hq, D = q.shape
    n_pages, Hk, page_size, _ = k_pool.shape
    dev, dtype = q.get_device(), q.dtype
    for x in (k_new, v_new):
        if x.dtype is not dtype or x.get_device() != dev or x.shape != (T, Hk, D):
            raise ValueError(f"{w}: k_new and v_new must be [T, Hk, D] in q's dtype, on its device")
    for x in (q, k_new, v_new):
        if x.stride(2) != 1 and x.numel():
            raise ValueError(f"{w}: head dimension must be contiguous")
    _expect(w, dev, "q_out", q_out, (T, Hq, D), dtype)
    _expect(w, dev, "k_pool", k_pool, (n_pages, Hk, page_size, D), dtype)
    _expect(w, dev, "v_pool", v_pool, (n_pages, Hk, page_size, D), dtype)
    _expect(w, dev, "wq", wq, (D,), dtype)
    _expect(w, dev, "wk", wk, (D,), dtype)
    _int32(w, dev, "slots", slots, T)
    _int32(w, dev, "positions", positions, T)
    _on_current(w, dev)
    rc = lib().loma_qk_norm_rope_append(q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), _addr(wq), _addr(wk), q_out.data_ptr(),
                                        k_pool.data_ptr(), v_pool.data_ptr(), slots.data_ptr(), positions.data_ptr(), T, Hq, Hk, D,
                                        page_size, n_pages, _strides(q, (0, 1)), _strides(k_new, (0, 1)), _strides(v_new, (0, 1)),
                                        _dtype_code(q), eps, theta_base, _raw_stream(stream, dev))
    _check(rc, w)


def loma_decode_shared_workspace_bytes(B: int, Hq: int, Hkv: int, D: int, prefix_len: int, max_cache_len: int) -> int:
    return int(lib().loma_decode_shared_workspace_bytes(B, Hq, Hkv, D, int(prefix_len), int(max_cache_len)))


def _shared_common(where, q, k_new, v_new, o, lse, cache_lens, Hkv, workspace):
    """Checks that both forms share; returns (device, dtype, B, Hq, D, workspace bytes)."""
    if q.dim() != 4 or q.shape[2] != 1 or not q.is_contiguous():
        raise ValueError(f"{where}: q must be a contiguous [B, Hq, 1, D] tensor")
    B, Hq, _, D = q.shape
    dev, dtype = q.get_device(), q.dtype
    _expect(where, dev, "o", o, q.shape, dtype)
    _expect(where, dev, "k_new", k_new, (B, Hkv, 1, D), dtype)
    _expect(where, dev, "v_new", v_new, (B, Hkv, 1, D), dtype)
    _expect(where, dev, "lse", lse, (B, Hq), torch.float32)
    _int32(where, dev, "cache_lens", cache_lens, B)
    return dev, dtype, B, Hq, D, _scratch(where, dev, workspace)


def loma_decode_attn_shared(q, k_new, v_new, k_prefix, v_prefix, prefix_len: int, k_cache, v_cache, o, lse, cache_lens,
                            max_cache_len: int, workspace=None, flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """Decode step over a prefix shared by the batch.  q, o: [B, Hq, 1, D]; k_new, v_new: [B, Hkv, 1, D] or None (already
    stored); k_prefix, v_prefix: [Hkv, prefix_cap, D]; own caches [B, Hkv, cap, D]; cache_lens: int32 [B], negative = no request;
    workspace: loma_decode_shared_workspace_bytes(...) bytes."""
    w = "loma_decode_attn_shared"
    Hkv, cap = k_cache.shape[1], k_cache.shape[2]
    dev, dtype, B, Hq, D, ws_bytes = _shared_common(w, q, k_new, v_new, o, lse, cache_lens, Hkv, workspace)
    _expect(w, dev, "k_cache", k_cache, (B, Hkv, cap, D), dtype)
    _expect(w, dev, "v_cache", v_cache, (B, Hkv, cap, D), dtype)
    prefix_cap = 0 if k_prefix is None else k_prefix.shape[1]
    _expect(w, dev, "k_prefix", k_prefix, (Hkv, prefix_cap, D), dtype)
    _expect(w, dev, "v_prefix", v_prefix, (Hkv, prefix_cap, D), dtype)
    _on_current(w, dev)
    rc = lib().loma_decode_attn_shared(q.data_ptr(), _addr(k_new), _addr(v_new), _addr(k_prefix), _addr(v_prefix), k_cache.data_ptr(),
                                       v_cache.data_ptr(), o.data_ptr(), _addr(lse), B, Hq, Hkv, D, prefix_cap, prefix_len, cap,
                                       cache_lens.data_ptr(), max_cache_len, _dtype_code(q), softmax_scale, flags, _addr(workspace),
                                       ws_bytes, _raw_stream(stream, dev))
    _check(rc, w)


def loma_decode_attn_shared_paged(q, k_new, v_new, k_pool, v_pool, prefix_table, prefix_len: int, block_table, o, lse, cache_lens,
                                  max_cache_len: int, workspace=None, flags: int = 0, softmax_scale: float = 0.0, stream=None) -> None:
    """loma_decode_attn_shared over a pool [n_pages, Hkv, page_size, D] that holds the prefix (prefix_table: int32
    [prefix_pages]) and the sequences' own entries (block_table: int32 [B, max_pages])."""
    w = "loma_decode_attn_shared_paged"
    n_pages, Hkv, page_size, _ = k_pool.shape
    dev, dtype, B, Hq, D, ws_bytes = _shared_common(w, q, k_new, v_new, o, lse, cache_lens, Hkv, workspace)
    _expect(w, dev, "k_pool", k_pool, (n_pages, Hkv, page_size, D), dtype)
    _expect(w, dev, "v_pool", v_pool, (n_pages, Hkv, page_size, D), dtype)
    _int32(w, dev, "prefix_table", prefix_table, -1)
    _int32(w, dev, "block_table", block_table, -1)
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError(f"{w}: block_table must be [B, max_pages]")
    _on_current(w, dev)
    rc = lib().loma_decode_attn_shared_paged(q.data_ptr(), _addr(k_new), _addr(v_new), k_pool.data_ptr(), v_pool.data_ptr(),
                                             _addr(prefix_table), block_table.data_ptr(), o.data_ptr(), _addr(lse), B, Hq, Hkv, D, page_size,
                                             0 if prefix_table is None else prefix_table.numel(), prefix_len, block_table.shape[1], n_pages,
                                             cache_lens.data_ptr(), max_cache_len, _dtype_code(q), softmax_scale, flags, _addr(workspace),
                                             ws_bytes, _raw_stream(stream, dev))
    _check(rc, w)
