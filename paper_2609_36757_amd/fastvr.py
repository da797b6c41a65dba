"""ctypes binding of libfastvr.so (declared in include/fastvr.h).

Argument marshalling only: every step of the computation runs in the HIP
kernels of the library.  torch tensors provide device memory and the stream.
If the library is missing, every call raises; there is no fallback."""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import NamedTuple

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libfastvr.so")

OK = 0
ERR_INVALID_ARGUMENT = 1
ERR_UNSUPPORTED = 2
ERR_CAPACITY = 3
ERR_HIP = 4

EXPORTED = ("fastvr_chunk_attn_fwd", "fastvr_chunk_attn_fwd_ex", "fastvr_kv_cache_append",
            "fastvr_chunk_attn_ring_step", "fastvr_chunk_attn_bwd", "fastvr_chunk_attn_bwd_noalloc",
            "fastvr_one_step_update",
            "fastvr_tile_axis", "fastvr_tile_gather", "fastvr_tile_blend", "fastvr_tile_blend_update",
            "fastvr_rope", "fastvr_kv4_append", "fastvr_kv4_read", "fastvr_kv4_attn_workspace", "fastvr_kv4_attn",
            "fastvr_status_string", "fastvr_last_error", "fastvr_abi_version")

_i64 = ctypes.c_int64
_vp = ctypes.c_void_p
_LIB = None


class FastVRError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


def load() -> ctypes.CDLL:
    """Load the in-tree libfastvr.so (built by ``python -m paper_2609_36757_amd.build``)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_36757_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    lib.fastvr_chunk_attn_fwd.restype = ctypes.c_int
    lib.fastvr_chunk_attn_fwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64, _i64, _i64,
                                          _i64, ctypes.c_float, _vp]
    lib.fastvr_chunk_attn_fwd_ex.restype = ctypes.c_int
    lib.fastvr_chunk_attn_fwd_ex.argtypes = [_vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64,
                                             ctypes.c_int32, _vp, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _i64,
                                             ctypes.c_float, _vp]
    lib.fastvr_kv_cache_append.restype = ctypes.c_int
    lib.fastvr_kv_cache_append.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64, _i64, _vp]
    lib.fastvr_chunk_attn_ring_step.restype = ctypes.c_int
    lib.fastvr_chunk_attn_ring_step.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64,
                                                _i64, _i64, ctypes.c_float, _vp]
    lib.fastvr_chunk_attn_bwd.restype = ctypes.c_int
    lib.fastvr_chunk_attn_bwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64,
                                          _i64, _i64, _i64, _i64, ctypes.c_float, _vp]
    lib.fastvr_chunk_attn_bwd_noalloc.restype = ctypes.c_int
    lib.fastvr_chunk_attn_bwd_noalloc.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64,
                                                  _i64, _i64, _i64, _i64, _i64, ctypes.c_float, _vp]
    lib.fastvr_one_step_update.restype = ctypes.c_int
    lib.fastvr_one_step_update.argtypes = [_vp, _vp, _vp, _i64, ctypes.c_float, ctypes.c_int32, _vp]
    lib.fastvr_tile_axis.restype = ctypes.c_int
    lib.fastvr_tile_axis.argtypes = [_i64, _i64, _i64, ctypes.POINTER(_i64), ctypes.POINTER(_i64)]
    lib.fastvr_tile_gather.restype = ctypes.c_int
    lib.fastvr_tile_gather.argtypes = [_vp, _vp, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _vp]
    lib.fastvr_tile_blend.restype = ctypes.c_int
    lib.fastvr_tile_blend.argtypes = [_vp, _vp, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _vp]
    lib.fastvr_tile_blend_update.restype = ctypes.c_int
    lib.fastvr_tile_blend_update.argtypes = [_vp, _vp, _vp, ctypes.c_float, _i64, _i64, _i64, _i64, _i64, _i64,
                                             _i64, _vp]
    _i32, _f64 = ctypes.c_int32, ctypes.c_double
    lib.fastvr_rope.restype = ctypes.c_int
    lib.fastvr_rope.argtypes = [_vp, _i64, _i64, _i32, _vp, _i64, _i64, _i32, _vp, _i64, _i64, _i64, _i64, _vp, _i64,
                                _f64, _i32, _i32, _i64, _i64, _i64, _i64, _vp]
    for copy in (lib.fastvr_kv4_append, lib.fastvr_kv4_read):
        copy.restype = ctypes.c_int
        copy.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _i64, _i64, _i64, _i64,
                         _vp]
    lib.fastvr_kv4_attn_workspace.restype = ctypes.c_int
    lib.fastvr_kv4_attn_workspace.argtypes = [_i64, _i64, _i64, _i64, _i64, _i64, _i64, _i64, ctypes.POINTER(_i64)]
    lib.fastvr_kv4_attn.restype = ctypes.c_int
    lib.fastvr_kv4_attn.argtypes = [_vp, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _vp, _vp, _i64, _vp,
                                    _i64, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _i64, ctypes.c_float, _vp]
    lib.fastvr_status_string.restype = ctypes.c_char_p
    lib.fastvr_status_string.argtypes = [ctypes.c_int]
    lib.fastvr_last_error.restype = ctypes.c_char_p
    lib.fastvr_last_error.argtypes = []
    lib.fastvr_abi_version.restype = ctypes.c_int
    lib.fastvr_abi_version.argtypes = []
    _LIB = lib
    return lib


def _check(status: int) -> None:
    if status != OK:
        lib = load()
        name = lib.fastvr_status_string(status).decode()
        detail = lib.fastvr_last_error().decode()
        raise FastVRError(status, f"{name}: {detail}")


def last_error() -> str:
    return load().fastvr_last_error().decode()


# ---------------------------------------------------------------------------
# raw entry points (integers for pointers; used by the tests and the bench)
# ---------------------------------------------------------------------------

def fwd_raw(q, k, v, o, lse, B, H, Nq, Nkv, d, chunk_len, q_chunk_offset, window_chunks, scale,
            stream=0) -> int:
    return load().fastvr_chunk_attn_fwd(q, k, v, o, lse, B, H, Nq, Nkv, d, chunk_len, q_chunk_offset,
                                        window_chunks, scale, stream)


def fwd_ex_raw(q, q_sb, q_st, k, k_sb, k_st, v, v_sb, v_st, o, o_sb, o_st, o_bf16, lse, B, H, Nq, Nkv, d,
               chunk_len, q_chunk_offset, window_chunks, scale, stream=0) -> int:
    return load().fastvr_chunk_attn_fwd_ex(q, q_sb, q_st, k, k_sb, k_st, v, v_sb, v_st, o, o_sb, o_st, o_bf16,
                                           lse, B, H, Nq, Nkv, d, chunk_len, q_chunk_offset, window_chunks,
                                           scale, stream)


def append_raw(k_cache, v_cache, k_new, v_new, B, H, d, capacity, cache_len, n_new, stream=0) -> int:
    return load().fastvr_kv_cache_append(k_cache, v_cache, k_new, v_new, B, H, d, capacity, cache_len,
                                         n_new, stream)


def ring_step_raw(q_new, k_new, v_new, k_ring, v_ring, o, lse, B, H, n_new, d, chunk_len, chunk_index,
                  window_chunks, scale, stream=0) -> int:
    return load().fastvr_chunk_attn_ring_step(q_new, k_new, v_new, k_ring, v_ring, o, lse, B, H, n_new, d,
                                              chunk_len, chunk_index, window_chunks, scale, stream)


def bwd_raw(q, k, v, o, lse, dout, dq, dk, dv, row_stats, B, H, Nq, Nkv, d, chunk_len, q_chunk_offset,
            window_chunks, scale, stream=0) -> int:
    return load().fastvr_chunk_attn_bwd(q, k, v, o, lse, dout, dq, dk, dv, row_stats, B, H, Nq, Nkv, d, chunk_len,
                                        q_chunk_offset, window_chunks, scale, stream)


def bwd_noalloc_raw(q, k, v, o, lse, dout, dq, dk, dv, B, H, Nq, Nkv, d, chunk_len, q_chunk_offset, window_chunks,
                    scale, stream=0) -> int:
    return load().fastvr_chunk_attn_bwd_noalloc(q, k, v, o, lse, dout, dq, dk, dv, B, H, Nq, Nkv, d, chunk_len,
                                                q_chunk_offset, window_chunks, scale, stream)


def one_step_raw(z_lq, v, z_hat, n, sigma, out_bf16, stream=0) -> int:
    return load().fastvr_one_step_update(z_lq, v, z_hat, n, sigma, out_bf16, stream)


def tile_axis(size: int, tile: int, overlap: int):
    """(number of tiles, tile length) along one axis, as the library places them."""
    n, L = _i64(0), _i64(0)
    _check(load().fastvr_tile_axis(size, tile, overlap, ctypes.byref(n), ctypes.byref(L)))
    return n.value, L.value


def tile_gather_raw(x, tiles, B, T, Hg, Wg, C, tile, overlap, stream=0) -> int:
    return load().fastvr_tile_gather(x, tiles, B, T, Hg, Wg, C, tile, overlap, stream)


def tile_blend_raw(tiles, out, B, T, Hg, Wg, C, tile, overlap, stream=0) -> int:
    return load().fastvr_tile_blend(tiles, out, B, T, Hg, Wg, C, tile, overlap, stream)


def tile_blend_update_raw(v_tiles, z_lq, z_hat, sigma, B, T, Hg, Wg, C, tile, overlap, stream=0) -> int:
    return load().fastvr_tile_blend_update(v_tiles, z_lq, z_hat, sigma, B, T, Hg, Wg, C, tile, overlap, stream)


def rope_raw(x, x_sb, x_st, x_fp32, y, y_sb, y_st, y_fp32, positions, pos_sb, n_axes, split1, split2, inv_freq, n_pairs,
             amplitude, interleaved, inverse, B, N, H, d, stream=0) -> int:
    return load().fastvr_rope(x, x_sb, x_st, x_fp32, y, y_sb, y_st, y_fp32, positions, pos_sb, n_axes, split1, split2,
                              inv_freq, n_pairs, amplitude, interleaved, inverse, B, N, H, d, stream)


def kv4_append_raw(k_codes, k_scales, v_codes, v_scales, k_new, k_sb, k_st, v_new, v_sb, v_st, starts, B, H, d, capacity,
                   first, n_new, stream=0) -> int:
    return load().fastvr_kv4_append(k_codes, k_scales, v_codes, v_scales, k_new, k_sb, k_st, v_new, v_sb, v_st, starts,
                                    B, H, d, capacity, first, n_new, stream)


def kv4_read_raw(k_codes, k_scales, v_codes, v_scales, k_out, k_sb, k_st, v_out, v_sb, v_st, starts, B, H, d, capacity,
                 first, n, stream=0) -> int:
    return load().fastvr_kv4_read(k_codes, k_scales, v_codes, v_scales, k_out, k_sb, k_st, v_out, v_sb, v_st, starts,
                                  B, H, d, capacity, first, n, stream)


def kv4_attn_workspace(B: int, H: int, Hkv: int, Nq: int, d: int, cache_len: int, chunk_len: int,
                       window_chunks: int = -1) -> int:
    """Bytes of device memory that a kv4_attn call of these sizes needs as its workspace."""
    n = _i64(0)
    _check(load().fastvr_kv4_attn_workspace(B, H, Hkv, Nq, d, cache_len, chunk_len, window_chunks, ctypes.byref(n)))
    return n.value


def kv4_attn_raw(q, q_sb, q_st, k_codes, k_scales, v_codes, v_scales, o, o_sb, o_st, o_bf16, lse, workspace,
                 workspace_bytes, lens, B, H, Hkv, Nq, d, capacity, cache_len, chunk_len, window_chunks, scale,
                 stream=0) -> int:
    return load().fastvr_kv4_attn(q, q_sb, q_st, k_codes, k_scales, v_codes, v_scales, o, o_sb, o_st, o_bf16, lse,
                                  workspace, workspace_bytes, lens, B, H, Hkv, Nq, d, capacity, cache_len, chunk_len,
                                  window_chunks, scale, stream)


# ---------------------------------------------------------------------------
# torch-facing wrappers
# ---------------------------------------------------------------------------

# The checks and allocations below are on the path of calls whose kernels take
# 5 to 20 us.  Measured on the host: torch.cuda.current_stream() 2.8 us against
# 0.1 us for its raw handle (two private functions of torch, so a torch without
# them takes the public way); torch.empty(..., device=...) 1.8 us against 1.3 to
# 1.6 us for empty_like / new_empty.

def _stream_handle(stream):
    if stream is not None:
        return stream.cuda_stream
    import torch
    try:
        raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream
    return raw(device())  # current stream of the current device


def _bnhd_strides(t, name):
    """(batch stride, token stride) of a [B, N, H, d] view whose heads and dims
    are packed (stride(3) == 1, stride(2) == d)."""
    if t.dim() != 4:
        raise ValueError(f"{name} must be 4-D [B, N, H, d]")
    if t.stride(3) != 1 or t.stride(2) != t.shape[3]:
        raise ValueError(f"{name}: heads and head_dim must be contiguous (stride(2) == d, stride(3) == 1)")
    return t.stride(0), t.stride(1)


def chunk_attn(q, k, v, *, chunk_len: int, q_chunk_offset: int = 0, window_chunks: int = -1,
               scale: float | None = None, out=None, lse=None, return_lse: bool = True, stream=None):
    """Chunk-causal attention forward (FastVR Sec. 3.1, Eq. 1).

    q [B, Nq, H, d], k/v [B, Nkv, H, d] bf16 GPU tensors (views allowed when
    heads and head_dim are packed).  Returns (o [B, Nq, H, d], lse fp32
    [B, H, Nq] or None); o is fp32 unless ``out`` is a bfloat16 tensor, which
    receives O rounded to bf16."""
    import torch
    bf16, fp32 = torch.bfloat16, torch.float32
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dtype != bf16 or not t.is_cuda:
            raise ValueError(f"{name} must be a bfloat16 GPU tensor")
    shape, kv_shape = q.shape, k.shape
    B, Nq, H, d = shape
    Nkv = kv_shape[1]
    if kv_shape != (B, Nkv, H, d) or v.shape != kv_shape:
        raise ValueError(f"shape mismatch: q {tuple(shape)} k {tuple(kv_shape)} v {tuple(v.shape)}")
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if out is None:
        out = q.new_empty(shape, dtype=fp32)
        o_bf16 = 0
    else:
        o_bf16 = 1 if out.dtype == bf16 else 0
        if not o_bf16 and out.dtype != fp32 or out.shape != shape:
            raise ValueError("out must be float32 or bfloat16 [B, Nq, H, d]")
    if lse is not None:
        if lse.dtype != fp32 or lse.shape != (B, H, Nq) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32 [B, H, Nq] tensor")
    elif return_lse:
        lse = q.new_empty((B, H, Nq), dtype=fp32)
    lse_ptr = lse.data_ptr() if lse is not None else None
    st = _stream_handle(stream)
    if not o_bf16 and q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and out.is_contiguous():
        status = load().fastvr_chunk_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse_ptr, B, H,
                                              Nq, Nkv, d, chunk_len, q_chunk_offset, window_chunks, scale, st)
    else:
        qs, ks, vs, os_ = (_bnhd_strides(t, n) for t, n in ((q, "q"), (k, "k"), (v, "v"), (out, "out")))
        status = fwd_ex_raw(q.data_ptr(), *qs, k.data_ptr(), *ks, v.data_ptr(), *vs, out.data_ptr(), *os_, o_bf16,
                            lse_ptr, B, H, Nq, Nkv, d, chunk_len, q_chunk_offset, window_chunks, scale, st)
    if status:
        _check(status)
    return out, lse


def kv_cache_append(k_cache, v_cache, k_new, v_new, cache_len: int, stream=None) -> int:
    """Copy k_new/v_new [B, n_new, H, d] into the contiguous caches [B, capacity, H, d]
    at token offset cache_len; returns the new cache length."""
    import torch
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache), ("k_new", k_new), ("v_new", v_new)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bfloat16 GPU tensor")
    B, cap, H, d = k_cache.shape
    n_new = k_new.shape[1]
    if v_cache.shape != k_cache.shape or k_new.shape != (B, n_new, H, d) or v_new.shape != k_new.shape:
        raise ValueError("cache / new-chunk shape mismatch")
    _check(append_raw(k_cache.data_ptr(), v_cache.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), B, H, d, cap,
                      cache_len, n_new, _stream_handle(stream)))
    return cache_len + n_new


def chunk_attn_ring_step(q_new, k_new, v_new, k_ring, v_ring, *, chunk_len: int, chunk_index: int,
                         window_chunks: int = 1, scale: float | None = None, out=None, lse=None,
                         return_lse: bool = True, stream=None):
    """One streaming step with a bounded ring KV cache of window_chunks + 1 chunk slots.

    q_new/k_new/v_new [B, n_new, H, d] bf16 hold chunk ``chunk_index`` of the
    stream; k_ring/v_ring [B, (window_chunks + 1) * chunk_len, H, d] bf16 hold
    the earlier chunks (chunk c in slot c mod (window_chunks + 1)).  The library
    writes the new chunk into its slot and returns (o fp32 [B, n_new, H, d],
    lse fp32 [B, H, n_new] or None) over chunks chunk_index - window_chunks ..
    chunk_index.  All tensors contiguous."""
    import torch
    for name, t in (("q_new", q_new), ("k_new", k_new), ("v_new", v_new), ("k_ring", k_ring), ("v_ring", v_ring)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bfloat16 GPU tensor")
    B, n_new, H, d = q_new.shape
    if k_new.shape != q_new.shape or v_new.shape != q_new.shape:
        raise ValueError("q_new, k_new and v_new must have the same shape")
    if k_ring.shape != (B, (window_chunks + 1) * chunk_len, H, d) or v_ring.shape != k_ring.shape:
        raise ValueError("k_ring/v_ring must be [B, (window_chunks + 1) * chunk_len, H, d]")
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if out is None:
        out = q_new.new_empty((B, n_new, H, d), dtype=torch.float32)
    if out.dtype != torch.float32 or tuple(out.shape) != (B, n_new, H, d) or not out.is_contiguous():
        raise ValueError("out must be a contiguous float32 [B, n_new, H, d] tensor")
    if return_lse and lse is None:
        lse = q_new.new_empty((B, H, n_new), dtype=torch.float32)
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (B, H, n_new)
                            or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 [B, H, n_new] tensor")
    _check(ring_step_raw(q_new.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), k_ring.data_ptr(), v_ring.data_ptr(),
                         out.data_ptr(), lse.data_ptr() if lse is not None else None, B, H, n_new, d, chunk_len,
                         chunk_index, window_chunks, scale, _stream_handle(stream)))
    return out, lse


def chunk_attn_bwd(q, k, v, o, lse, dout, *, chunk_len: int, q_chunk_offset: int = 0, window_chunks: int = -1,
                   scale: float | None = None, dq=None, dk=None, dv=None, row_stats=None, stream=None):
    """Gradients (dq, dk, dv), fp32, of chunk_attn for the upstream gradient ``dout``.

    q/dout [B, Nq, H, d] and k/v [B, Nkv, H, d] bf16, o fp32 [B, Nq, H, d] and
    lse fp32 [B, H, Nq] from the forward call with the same mask arguments and
    scale; all contiguous.  ``row_stats`` (fp32 [B, H, 2, Nq]) is a workspace the
    call fills with LSE * log2 e (plane 0) and -rowsum(dO * O) (plane 1)."""
    import torch
    for name, t in (("q", q), ("k", k), ("v", v), ("dout", dout)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bfloat16 GPU tensor")
    B, Nq, H, d = q.shape
    Nkv = k.shape[1]
    if k.shape != (B, Nkv, H, d) or v.shape != k.shape or dout.shape != q.shape:
        raise ValueError(f"shape mismatch: q {tuple(q.shape)} k {tuple(k.shape)} v {tuple(v.shape)} "
                         f"dout {tuple(dout.shape)}")
    for name, t, shape in (("o", o, (B, Nq, H, d)), ("lse", lse, (B, H, Nq))):
        if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 {list(shape)} tensor")
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    outs = []
    for name, t, shape in (("dq", dq, (B, Nq, H, d)), ("dk", dk, (B, Nkv, H, d)), ("dv", dv, (B, Nkv, H, d)),
                           ("row_stats", row_stats, (B, H, 2, Nq))):
        if t is None:
            t = q.new_empty(shape, dtype=torch.float32)
        elif t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 {list(shape)} tensor")
        outs.append(t)
    dq, dk, dv, row_stats = outs
    _check(bwd_raw(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
                   dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), row_stats.data_ptr(), B, H, Nq, Nkv, d, chunk_len,
                   q_chunk_offset, window_chunks, scale, _stream_handle(stream)))
    return dq, dk, dv


def chunk_attn_bwd_noalloc(q, k, v, o, lse, dout, dq, dk, dv, *, chunk_len: int, q_chunk_offset: int = 0,
                           window_chunks: int = -1, scale: float | None = None, stream=None):
    """chunk_attn_bwd for callers that cannot allocate: the caller passes the
    outputs dq, dk, dv (fp32, contiguous, shapes as in chunk_attn_bwd) and the
    row statistics go to the library's static per-device workspace, so neither
    the library nor this binding allocates.  Calls that overlap in time on one
    device race on that workspace."""
    import torch
    for name, t in (("q", q), ("k", k), ("v", v), ("dout", dout)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bfloat16 GPU tensor")
    B, Nq, H, d = q.shape
    Nkv = k.shape[1]
    if k.shape != (B, Nkv, H, d) or v.shape != k.shape or dout.shape != q.shape:
        raise ValueError(f"shape mismatch: q {tuple(q.shape)} k {tuple(k.shape)} v {tuple(v.shape)} "
                         f"dout {tuple(dout.shape)}")
    for name, t, shape in (("o", o, (B, Nq, H, d)), ("lse", lse, (B, H, Nq)), ("dq", dq, (B, Nq, H, d)),
                           ("dk", dk, (B, Nkv, H, d)), ("dv", dv, (B, Nkv, H, d))):
        if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 {list(shape)} tensor")
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    _check(bwd_noalloc_raw(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
                           dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Nq, Nkv, d, chunk_len, q_chunk_offset,
                           window_chunks, scale, _stream_handle(stream)))
    return dq, dk, dv


def one_step_update(z_lq, v, sigma: float, *, out=None, out_dtype=None, stream=None):
    """One-step latent update z_hat = z_lq - sigma * v (FastVR Eq. 9).

    z_lq, v: contiguous bf16 GPU tensors of one shape.  The result is float32
    (default) or bfloat16 (``out_dtype=torch.bfloat16``; ``out`` may then be
    z_lq or v itself, for an update in place)."""
    import torch
    for name, t in (("z_lq", z_lq), ("v", v)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bfloat16 GPU tensor")
    if v.shape != z_lq.shape:
        raise ValueError(f"shape mismatch: z_lq {tuple(z_lq.shape)} v {tuple(v.shape)}")
    if out_dtype is None:
        out_dtype = out.dtype if out is not None else torch.float32
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be float32 or bfloat16")
    if out is None:
        out = z_lq.new_empty(z_lq.shape, dtype=out_dtype)
    elif out.dtype != out_dtype or out.shape != z_lq.shape or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of z_lq's shape and dtype out_dtype")
    _check(one_step_raw(z_lq.data_ptr(), v.data_ptr(), out.data_ptr(), z_lq.numel(), sigma,
                        1 if out_dtype == torch.bfloat16 else 0, _stream_handle(stream)))
    return out


# a pure function of three integers; typed, so that what tile_axis refuses stays refused
_axis = functools.lru_cache(maxsize=64, typed=True)(tile_axis)


def _tile_shape(B, T, Hg, Wg, C, tile, overlap):
    ny, Ly = _axis(Hg, tile, overlap)
    nx, Lx = _axis(Wg, tile, overlap)
    return (B, ny * nx, T, Ly, Lx, C)


def tile_gather(x, *, tile: int = 64, overlap: int = 16, out=None, stream=None):
    """Overlapping spatial tiles of a channels-last bf16 field x [B, T, Hg, Wg, C]
    -> [B, ny * nx, T, Ly, Lx, C] (placement as in include/fastvr.h)."""
    import torch
    if x.dtype != torch.bfloat16 or not x.is_cuda or not x.is_contiguous() or x.dim() != 5:
        raise ValueError("x must be a contiguous bfloat16 GPU tensor [B, T, Hg, Wg, C]")
    B, T, Hg, Wg, C = x.shape
    shape = _tile_shape(B, T, Hg, Wg, C, tile, overlap)
    if out is None:
        out = x.new_empty(shape)
    elif out.dtype != torch.bfloat16 or tuple(out.shape) != shape or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous bfloat16 tensor of shape {shape}")
    _check(tile_gather_raw(x.data_ptr(), out.data_ptr(), B, T, Hg, Wg, C, tile, overlap, _stream_handle(stream)))
    return out


def tile_blend(tiles, Hg: int, Wg: int, *, tile: int = 64, overlap: int = 16, z_lq=None, sigma: float = 0.0,
               out=None, stream=None):
    """Weight-normalised blend of fp32 tiles [B, ny * nx, T, Ly, Lx, C] into the
    field [B, T, Hg, Wg, C] (fp32).  With z_lq (bf16 [B, T, Hg, Wg, C]) the result
    is the one-step update z_lq - sigma * blend (Eq. 9), fused."""
    import torch
    if tiles.dtype != torch.float32 or not tiles.is_cuda or not tiles.is_contiguous() or tiles.dim() != 6:
        raise ValueError("tiles must be a contiguous float32 GPU tensor [B, ny*nx, T, Ly, Lx, C]")
    B, _, T, _, _, C = tiles.shape
    if tuple(tiles.shape) != _tile_shape(B, T, Hg, Wg, C, tile, overlap):
        raise ValueError("tiles do not match the grid, tile and overlap")
    shape = (B, T, Hg, Wg, C)
    if out is None:
        out = tiles.new_empty(shape)
    elif out.dtype != torch.float32 or tuple(out.shape) != shape or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous float32 tensor of shape {shape}")
    st = _stream_handle(stream)
    if z_lq is None:
        _check(tile_blend_raw(tiles.data_ptr(), out.data_ptr(), B, T, Hg, Wg, C, tile, overlap, st))
    else:
        if z_lq.dtype != torch.bfloat16 or tuple(z_lq.shape) != shape or not z_lq.is_contiguous():
            raise ValueError(f"z_lq must be a contiguous bfloat16 tensor of shape {shape}")
        _check(tile_blend_update_raw(tiles.data_ptr(), z_lq.data_ptr(), out.data_ptr(), sigma, B, T, Hg, Wg, C, tile,
                                     overlap, st))
    return out


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

# The checks below are on the path of calls whose kernels take 3 to 10 us, so the usual
# case is decided with few calls into torch (0.05 to 0.1 us each): contiguous tensors, one device.

def _view_strides(t, name, shape):
    """_bnhd_strides, of a view of that shape, with the strides of axes of one element, which
    torch leaves to chance, as if the view were contiguous there."""
    B, N, H, d = shape
    if t.is_contiguous():
        return N * H * d, H * d
    sb, st, sh, sd = t.stride()
    if sd != 1 and d != 1 or sh != d and H != 1:
        raise ValueError(f"{name}: heads and head_dim must be contiguous (stride(2) == d, stride(3) == 1)")
    if N == 1:
        st = H * d
    if B == 1:
        sb = N * st
    return sb, st


def _check_view(t, name, shape, dtype):
    """Strides of a [B, N, H, d] view of that shape (None: its own, known to have four axes) and dtype."""
    if t.dtype is not dtype or not t.is_cuda:
        raise ValueError(f"{name} must be a {str(dtype).split('.')[1]} GPU tensor")
    if shape is None:
        shape = t.shape
    elif t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return _view_strides(t, name, shape)


def _stream_on(device: int, stream, *tensors):
    """Handle of the stream that takes a call on the tensors (None: not given): the given one, or the
    current one of the current device, which all tensors have to be on."""
    import torch
    try:
        current = torch._C._cuda_getDevice()
        handle = torch._C._cuda_getCurrentRawStream(current) if stream is None else stream.cuda_stream
    except AttributeError:  # (as in _stream_handle)
        current = torch.cuda.current_device()
        handle = _stream_handle(stream)
    if device != current:
        raise ValueError(f"the tensors are on cuda:{device}, the current device is cuda:{current}")
    if stream is not None and getattr(stream, "device_index", device) != device:
        raise ValueError(f"the tensors are on cuda:{device}, the stream is on cuda:{stream.device_index}")
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"all tensors must be on cuda:{device}, one is on {t.device}")
    return handle


def _empty(like, shape, dtype, stream=None):
    """A contiguous tensor on like's device, for the stream that takes the call: torch's allocator hands
    memory out and takes it back in the order of one stream, and a workspace made here goes back
    as soon as the call has returned."""
    if stream is not None:
        import torch
        with torch.cuda.stream(stream):
            return like.new_empty(shape, dtype=dtype)
    return like.new_empty(shape, dtype=dtype)


def _empty_as(like, shape, dtype, stream):
    """_empty of like's own shape (empty_like: 1.1 us against 1.5)."""
    if stream is None and like.dtype is dtype and like.is_contiguous():
        import torch
        return torch.empty_like(like)
    return _empty(like, shape, dtype, stream)


def rope_inv_freq(n_pairs: int, *, base: float = 10000.0, sections=None, scaling: str | None = None,
                  factor: float = 1.0, original_len: int = 0, fast: float = 32.0, slow: float = 1.0):
    """(radians per position of each pair, amplitude) for ``rope``, as a list of floats and a float.

    Pair j of n turns by base^(-j / n) a position.  With ``sections`` (pairs per axis,
    for positions of several axes) each axis has frequencies of its own, j and n
    counted within it.  ``scaling``, for contexts ``factor`` times as long as the
    ``original_len`` positions that a model was trained on (one axis):

    * ``"linear"``: every frequency divided by ``factor``;
    * ``"ntk"``: base * factor^(n / (n - 1)), which keeps the fastest pair and divides the slowest by ``factor``;
    * ``"yarn"`` (arXiv 2309.00071): pairs that turn ``fast`` times or more within original_len
      are kept, those that turn ``slow`` times or less divided by ``factor``, the ones between
      blended linearly in their turns; amplitude 0.1 ln(factor) + 1; factor >= 1."""
    if n_pairs < 0 or not base > 0 or not factor > 0:
        raise ValueError("need n_pairs >= 0, base > 0 and factor > 0")
    if sections is not None:
        if scaling is not None:
            raise ValueError("scaling is for positions of one axis")
        if sum(sections) != n_pairs or min(sections) < 0:
            raise ValueError(f"sections {tuple(sections)} do not add up to {n_pairs} pairs")
        return [base ** (-j / n) for n in sections for j in range(n)], 1.0
    if scaling not in (None, "linear", "ntk", "yarn"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if scaling == "ntk":
        base *= factor ** (n_pairs / max(1, n_pairs - 1))
    freq = [base ** (-j / n_pairs) for j in range(n_pairs)]
    if scaling == "linear":
        return [f / factor for f in freq], 1.0
    if scaling == "yarn":
        if original_len < 1 or not fast > slow or not 1 <= factor < math.inf:
            raise ValueError("yarn needs original_len >= 1, fast > slow and a finite factor >= 1")
        keep = [min(1.0, max(0.0, (original_len * f / (2 * math.pi) - slow) / (fast - slow))) for f in freq]
        return [f * k + f / factor * (1 - k) for f, k in zip(freq, keep)], 0.1 * math.log(factor) + 1.0
    return freq, 1.0


def _rope(x, positions, inv_freq, layout, sections, amplitude, out, out_dtype, inverse, stream):
    import torch
    bf16, fp32 = torch.bfloat16, torch.float32
    if x.dim() != 4:
        raise ValueError("x must be 4-D [B, N, H, d]")
    shape = x.shape
    B, N, H, d = shape
    x32 = x.dtype is fp32
    xs = _check_view(x, "x", None, fp32 if x32 else bf16)
    if layout not in ("interleaved", "half"):
        raise ValueError(f"layout must be 'interleaved' or 'half', got {layout!r}")
    if inv_freq.dtype is not torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq must be a contiguous float64 tensor [pairs]")
    n_pairs = inv_freq.shape[0]
    A, split1, split2 = 1, n_pairs, n_pairs
    if sections is not None:
        A = len(sections)
        if not 1 <= A <= 3 or sum(sections) != n_pairs or min(sections) < 0:
            raise ValueError(f"sections {sections} must be one to three numbers of pairs that add up to {n_pairs}")
        split1 = sections[0]
        if A == 3:
            split2 = split1 + sections[1]
    if positions.dtype is not torch.int32 or not positions.is_contiguous():
        raise ValueError("positions must be a contiguous int32 tensor")
    ps = positions.shape
    if ps == (N, A) or A == 1 and ps == (N,):
        pos_sb = 0
    elif ps == (B, N, A) or A == 1 and ps == (B, N):
        pos_sb = N * A
    else:
        raise ValueError(f"positions must be [N, {A}] or [B, N, {A}], got {list(ps)}")
    if out_dtype is None:
        out_dtype = out.dtype if out is not None else x.dtype
    if out_dtype is not bf16 and out_dtype is not fp32:
        raise ValueError("out_dtype must be float32 or bfloat16")
    handle = _stream_on(x.get_device(), stream, positions, inv_freq, out)
    ys = (N * H * d, H * d)
    if out is None:
        out = _empty_as(x, shape, out_dtype, stream)
    else:
        ys = _check_view(out, "out", shape, out_dtype)
    status = load().fastvr_rope(x.data_ptr(), *xs, 1 if x32 else 0, out.data_ptr(), *ys,
                                1 if out_dtype is fp32 else 0, positions.data_ptr(), pos_sb, A, split1, split2,
                                inv_freq.data_ptr(), n_pairs, amplitude, 1 if layout == "interleaved" else 0, inverse,
                                B, N, H, d, handle)
    if status:
        _check(status)
    return out


def rope(x, positions, inv_freq, *, layout: str = "interleaved", sections=None, amplitude: float = 1.0, out=None,
         out_dtype=None, stream=None):
    """Rotary positions of the heads x [B, N, H, d] (bf16 or fp32; views as in chunk_attn, so
    q and k of a packed projection take one call).  Here and in the calls below, tensors that are
    not given are allocated for ``stream``, as under ``torch.cuda.stream``.

    ``inv_freq`` (float64 GPU tensor [pairs]) holds each pair's radians per position: the
    first 2 * pairs elements of a head turn, the others pass.  Pairs are neighbours (``layout="interleaved"``)
    or elements p and pairs + p (``"half"``).  ``positions`` (int32, [N, axes] or [B, N, axes]; [N]
    or [B, N] for one axis) are the tokens' positions; with ``sections`` (up to three numbers of
    pairs) the first section turns with axis 0, the next with axis 1 and so on: frame, row
    and column of a video token.  The result has x's dtype unless ``out`` or ``out_dtype`` says otherwise;
    ``out`` may be x itself."""
    return _rope(x, positions, inv_freq, layout, sections, amplitude, out, out_dtype, 0, stream)


def rope_bwd(dy, positions, inv_freq, *, layout: str = "interleaved", sections=None, amplitude: float = 1.0, out=None,
             out_dtype=None, stream=None):
    """Gradient of ``rope`` with respect to x, for the upstream gradient ``dy``: the turn by the
    negative angles.  Arguments as in ``rope``; dq and dk of chunk_attn_bwd (fp32) go in as they are."""
    return _rope(dy, positions, inv_freq, layout, sections, amplitude, out, out_dtype, 1, stream)


# ---------------------------------------------------------------------------
# KV cache in 4 bits
# ---------------------------------------------------------------------------

class KV4Cache(NamedTuple):
    """A KV cache in 4 bits: codes [B, H, capacity, d / 2] and scales [B, H, capacity, d / 32] (uint8)
    of keys and values; 0.53 bytes an element (the format is in include/fastvr.h)."""
    k_codes: object
    k_scales: object
    v_codes: object
    v_scales: object


def kv4_cache(B: int, capacity: int, H: int, d: int, device="cuda") -> KV4Cache:
    """An empty cache (zeros)."""
    import torch
    return KV4Cache(*(torch.zeros((B, H, capacity, n), dtype=torch.uint8, device=device)
                      for n in (d // 2, d // 32, d // 2, d // 32)))


def _check_kv4(cache):
    """(B, H, capacity, d) of a cache."""
    import torch
    u8 = torch.uint8
    kc, ks, vc, vs = cache
    for t in cache:
        if t.dtype is not u8 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("a 4-bit cache is four contiguous uint8 GPU tensors")
    shape = kc.shape
    if len(shape) != 4:
        raise ValueError("cache codes must be [B, H, capacity, d / 2]")
    B, H, cap, half = shape
    scales = (B, H, cap, half // 16)
    if vc.shape != shape or ks.shape != scales or vs.shape != scales:
        raise ValueError("cache shape mismatch: codes [B, H, capacity, d / 2], scales [B, H, capacity, d / 32]")
    return B, H, cap, 2 * half


def _check_int32(t, name, n):
    if t is None:
        return None
    import torch
    if t.dtype != torch.int32 or not t.is_cuda or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 GPU tensor [{n}]")
    return t.data_ptr()


def kv4_append(cache, k_new, v_new, cache_len: int = 0, *, starts=None, stream=None):
    """Quantise k_new/v_new [B, n_new, H, d] (bf16 views) into token rows cache_len .. of the
    cache and return the new cache length.  With ``starts`` (int32 GPU tensor [B]) sequence b's rows
    start at starts[b] instead, rows outside the cache are dropped, and None is returned."""
    import torch
    B, H, cap, d = _check_kv4(cache)
    if k_new.dim() != 4:
        raise ValueError("k_new must be 4-D [B, n_new, H, d]")
    n = k_new.shape[1]
    shape = (B, n, H, d)
    ks = _check_view(k_new, "k_new", shape, torch.bfloat16)
    vs = _check_view(v_new, "v_new", shape, torch.bfloat16)
    sp = _check_int32(starts, "starts", B)
    handle = _stream_on(k_new.get_device(), stream, v_new, *cache, starts)
    status = load().fastvr_kv4_append(*(t.data_ptr() for t in cache), k_new.data_ptr(), *ks, v_new.data_ptr(), *vs, sp,
                                      B, H, d, cap, cache_len, n, handle)
    if status:
        _check(status)
    return cache_len + n if starts is None else None


def kv4_read(cache, n: int, first: int = 0, *, starts=None, k_out=None, v_out=None, stream=None):
    """The values (k, v), bf16 [B, n, H, d], that the cache holds for n token rows from ``first``
    on, or from starts[b] (int32 GPU tensor [B]) of each sequence b; rows outside the cache are then zero."""
    import torch
    B, H, cap, d = _check_kv4(cache)
    shape = (B, n, H, d)
    contiguous = (n * H * d, H * d)
    ks = vs = contiguous
    if k_out is None:
        k_out = _empty(cache[0], shape, torch.bfloat16, stream)
    else:
        ks = _check_view(k_out, "k_out", shape, torch.bfloat16)
    if v_out is None:
        v_out = _empty_as(k_out, shape, torch.bfloat16, stream)
    else:
        vs = _check_view(v_out, "v_out", shape, torch.bfloat16)
    sp = _check_int32(starts, "starts", B)
    handle = _stream_on(k_out.get_device(), stream, v_out, *cache, starts)
    status = load().fastvr_kv4_read(*(t.data_ptr() for t in cache), k_out.data_ptr(), *ks, v_out.data_ptr(), *vs, sp, B,
                                    H, d, cap, first, n, handle)
    if status:
        _check(status)
    return k_out, v_out


# a pure function of integers; typed, so that what it refuses stays refused
_kv4_workspace = functools.lru_cache(maxsize=256, typed=True)(kv4_attn_workspace)


def kv4_attn(q, cache, cache_len: int, *, lens=None, chunk_len: int | None = None, window_chunks: int = -1,
             scale: float | None = None, out=None, out_dtype=None, lse=None, return_lse: bool = True, workspace=None,
             stream=None):
    """Attention of the newest Nq tokens, q [B, Nq, H, d] (bf16 view), over a 4-bit cache whose
    sequences hold cache_len tokens each, or lens[b] (int32 GPU tensor [B], at most cache_len).

    Row i is the token at position length - Nq + i and sees the chunks of chunk_len tokens
    up to its own one, window_chunks of them before it (-1: all); chunk_len None: the whole
    cache, 1: the tokens up to its own.  H may be a multiple of the cache's heads: query head h
    reads key head h // (H / Hkv).  Returns (o [B, Nq, H, d], float32 unless ``out`` or ``out_dtype`` says
    bfloat16, lse fp32 [B, H, Nq] or None).  Rows that see nothing: o = 0, lse = -inf.
    ``workspace``: a uint8 GPU tensor of kv4_attn_workspace(...) bytes, allocated here if None; two calls
    that may run at the same time need two."""
    import torch
    bf16, fp32 = torch.bfloat16, torch.float32
    B, Hkv, cap, d = _check_kv4(cache)
    if q.dim() != 4:
        raise ValueError("q must be 4-D [B, Nq, H, d]")
    shape = q.shape
    _, Nq, H, _ = shape
    if shape[0] != B or shape[3] != d:
        raise ValueError(f"shape mismatch: q {tuple(shape)}, cache of {B} sequences and head_dim {d}")
    qs = _check_view(q, "q", None, bf16)
    if chunk_len is None:
        chunk_len = max(cache_len, 1)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if out_dtype is None:
        out_dtype = out.dtype if out is not None else fp32
    if out_dtype is not bf16 and out_dtype is not fp32:
        raise ValueError("out_dtype must be float32 or bfloat16")
    handle = _stream_on(q.get_device(), stream, *cache, lens, out, lse, workspace)
    os_ = (Nq * H * d, H * d)
    if out is None:
        out = _empty_as(q, shape, out_dtype, stream)
    else:
        os_ = _check_view(out, "out", shape, out_dtype)
    if lse is not None:
        if lse.dtype != fp32 or lse.shape != (B, H, Nq) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32 [B, H, Nq] tensor")
    elif return_lse:
        lse = _empty(q, (B, H, Nq), fp32, stream)
    lp = _check_int32(lens, "lens", B)
    n_ws = _kv4_workspace(B, H, Hkv, Nq, d, cache_len, chunk_len, window_chunks)
    if workspace is None:
        if n_ws:
            workspace = _empty(q, (n_ws,), torch.uint8, stream)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor")
    else:
        n_ws = workspace.numel()
    status = load().fastvr_kv4_attn(q.data_ptr(), *qs, *(t.data_ptr() for t in cache), out.data_ptr(), *os_,
                                    1 if out_dtype is bf16 else 0, lse.data_ptr() if lse is not None else None,
                                    workspace.data_ptr() if workspace is not None else None, n_ws, lp, B, H, Hkv, Nq, d,
                                    cap, cache_len, chunk_len, window_chunks, scale, handle)
    if status:
        _check(status)
    return out, lse
