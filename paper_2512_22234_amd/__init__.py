"""bd_attn: block-diffusion masked attention for MI355X (gfx950).

Thin Python binding over the C-ABI library libbd_attn.so: the functions here
carry the names of the C entry points and only marshal arguments (shape and
dtype checks, output/workspace allocation through torch, the current HIP
stream).  Every step of the computation runs in the library's HIP kernels.

Attention over the packed sequence [x_t | x_0] of 2L tokens with the
block-diffusion mask of DiRL (arXiv 2512.22234, Section 4.1; Eq. 1 and
Eq. 2): a noisy query sees noisy keys of its own block and clean keys of
earlier blocks; a clean query sees clean keys of its own and earlier blocks.
"""
from __future__ import annotations

import collections
import contextlib
import ctypes
import functools
import operator

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from ._lib import LIB_PATH, BdAttnError, lib, status_string  # noqa: F401

BD_ATTN_BF16 = 0
BD_ATTN_FP32 = 1

__all__ = [
    "bd_attn", "BdAttnFunction", "bd_attn_fwd", "bd_attn_bwd", "bd_attn_workspace_bytes",
    "bd_attn_classify_tiles_host", "bd_attn_visit_lists_host", "bd_attn_mask_windows_host",
    "bd_attn_status_string", "bd_attn_bwd_noalloc", "BD_ATTN_NOALLOC_SCRATCH_BYTES",
    "bd_attn_version", "bd_attn_fwd_marked", "bd_attn_bwd_marked", "bd_attn_stage_names",
    "BdAttnError", "BD_ATTN_BF16", "BD_ATTN_FP32",
    "bd_attn_varlen", "BdAttnVarlenFunction", "bd_attn_varlen_fwd", "bd_attn_varlen_bwd",
    "bd_attn_varlen_workspace_bytes", "bd_attn_decode_fwd", "bd_attn_decode_workspace_bytes",
    "bd_lce_fwd", "bd_lce_bwd", "bd_lce_workspace_bytes", "bd_lce_logits_bytes", "bd_lce_objective", "LceFunction", "lm_head_logprobs",
    "BD_LCE_CE", "BD_LCE_DIPO",
    "bd_rope_table", "bd_qk_norm_rope_fwd", "bd_qk_norm_rope_bwd", "bd_qk_norm_rope_workspace_bytes",
    "QkNormRopeFunction", "QkvNormRopeFunction", "qk_norm_rope", "qkv_norm_rope", "bd_qk_norm_rope_paged",
    "bd_paged_plan", "PagedPlan", "bd_attn_paged_decode_fwd", "bd_attn_paged_decode_workspace_bytes",
    "bd_attn_paged_shared_decode_fwd", "bd_attn_paged_shared_decode_workspace_bytes", "bd_paged_summarize",
    "bd_paged_select", "bd_paged_select_workspace_bytes", "PagedLists", "bd_attn_paged_sparse_decode_fwd",
    "bd_attn_paged_sparse_decode_workspace_bytes",
]


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BD_ATTN_BF16
    if t.dtype == torch.float32:
        return BD_ATTN_FP32
    raise TypeError(f"bd_attn supports bfloat16 and float32 tensors, got {t.dtype}")


# The binding's own time is most of a small call (one sequence's decoding step:
# 19 us a call around 12 us of kernels), so pointers go to the library as plain
# integers, sizes that depend on the shape alone are looked up once per shape,
# and a tensor that passes all its checks is tested in one expression.

_ptr = torch.Tensor.data_ptr


def _stream_handle(device: torch.device, stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    # (a torch internal that saves building a Stream object, 1 us; not every build need have it)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None or device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return raw(device.index)


def _workspace(nbytes: int, device: torch.device, workspace):
    """The caller's workspace or a new one, and its pointer and size (none for 0 bytes)."""
    if workspace is not None:
        if workspace.device != device or not workspace.is_contiguous():
            raise ValueError(f"workspace: a contiguous tensor on {device} expected, got one on {workspace.device}")
        return workspace, workspace.data_ptr(), workspace.numel()
    if nbytes == 0:
        return None, None, 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), nbytes


def _check(name: str, t: torch.Tensor, shape, dtype, device):
    if t.shape == shape and t.dtype is dtype and t.device == device and t.is_contiguous():
        return
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: expected device {device}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")


def _query_size(name: str, *args) -> int:
    """The library's size function `name` (a function of the shape alone)."""
    return int(getattr(lib(), name)(*args))


_known_size = functools.lru_cache(maxsize=1024)(_query_size)


def _size(a, b):
    """The function that finds a call's size from the caller's own arguments a
    and b (the rest come from tensor shapes): only plain integers are looked
    up.  A NumPy or torch scalar may change its value in place, and need not be
    hashable."""
    return _known_size if type(a) is int and type(b) is int else _query_size


def _scale_arg(scale) -> float:
    return 0.0 if scale is None else float(scale)


def bd_attn_version() -> int:
    return int(lib().bd_attn_version())


def bd_attn_status_string(status: int) -> str:
    return status_string(status)


def bd_attn_workspace_bytes(B, L, S, Hq, Hkv, D, dtype, for_bwd) -> int:
    return int(lib().bd_attn_workspace_bytes(B, L, S, Hq, Hkv, D, int(dtype), int(for_bwd)))


def bd_attn_classify_tiles_host(L: int, S: int, BM: int, BN: int) -> np.ndarray:
    nq, nk = 2 * (-(-L // BM)), 2 * (-(-L // BN))
    out = np.zeros((nq, nk), dtype=np.int8)
    st = lib().bd_attn_classify_tiles_host(L, S, BM, BN, out.ctypes.data_as(ctypes.c_void_p))
    if st:
        raise BdAttnError(st, "bd_attn_classify_tiles_host")
    return out


def bd_attn_visit_lists_host(L: int, S: int, BM: int, BN: int, by_key_tile: bool, nsplit: int = 2) -> np.ndarray:
    nq, nk = 2 * (-(-L // BM)), 2 * (-(-L // BN))
    out = np.zeros((nq, nk), dtype=np.int8)
    st = lib().bd_attn_visit_lists_host(L, S, BM, BN, int(by_key_tile), nsplit, out.ctypes.data_as(ctypes.c_void_p))
    if st:
        raise BdAttnError(st, "bd_attn_visit_lists_host")
    return out


def bd_attn_mask_windows_host(L: int, S: int, by_key: bool) -> np.ndarray:
    out = np.zeros((2 * L, 2 * L), dtype=np.int8)
    st = lib().bd_attn_mask_windows_host(L, S, int(by_key), out.ctypes.data_as(ctypes.c_void_p))
    if st:
        raise BdAttnError(st, "bd_attn_mask_windows_host")
    return out


def bd_attn_group_windows_host(L: int, S: int, by_key: bool, group: int) -> np.ndarray:
    out = np.zeros((2 * L, 2 * L), dtype=np.int8)
    st = lib().bd_attn_group_windows_host(L, S, int(by_key), group, out.ctypes.data_as(ctypes.c_void_p))
    if st:
        raise BdAttnError(st, "bd_attn_group_windows_host")
    return out


def _shapes(q, k, L):
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q [B,Hq,2L,D] and k/v [B,Hkv,2L,D] expected")
    B, Hq, N, D = q.shape
    Hkv = k.shape[1]
    if N != 2 * L:
        raise ValueError(f"packed length {N} != 2L = {2 * L}")
    return B, Hq, Hkv, D


def _marks_arg(marks):
    """ctypes array of raw HIP event handles from torch.cuda.Event objects."""
    if not marks:
        return None, 0
    for ev in marks:
        if ev.cuda_event == 0:      # torch creates the event lazily on first record
            ev.record()
    arr = (ctypes.c_void_p * len(marks))(*[ev.cuda_event for ev in marks])
    return arr, len(marks)


def bd_attn_stage_names(for_bwd: bool, dtype: int = BD_ATTN_BF16):
    return lib().bd_attn_stage_names(int(for_bwd), int(dtype)).decode().split(",")


def bd_attn_fwd_marked(q, k, v, L: int, S: int, marks, scale=None, out=None, lse=None, workspace=None,
                       stream=None):
    """bd_attn_fwd that also records marks[2i] and marks[2i + 1] as kernel i begins and ends."""
    return bd_attn_fwd(q, k, v, L, S, scale, out, lse, workspace, stream, _marks=marks)


def bd_attn_bwd_marked(do, q, k, v, o, lse, L: int, S: int, marks, scale=None, dq=None, dk=None, dv=None,
                       workspace=None, stream=None):
    """bd_attn_bwd that also records marks[2i] and marks[2i + 1] as kernel i begins and ends."""
    return bd_attn_bwd(do, q, k, v, o, lse, L, S, scale, dq, dk, dv, workspace, stream, _marks=marks)


def bd_attn_fwd(q, k, v, L: int, S: int, scale=None, out=None, lse=None, workspace=None, stream=None,
                _marks=None):
    """Forward pass; returns (O, LSE).  O has q's dtype, LSE is float32 [B,Hq,2L]."""
    B, Hq, Hkv, D = _shapes(q, k, L)
    dev, dt = q.device, q.dtype
    code = _dtype_code(q)
    _check("q", q, (B, Hq, 2 * L, D), dt, dev)
    _check("k", k, (B, Hkv, 2 * L, D), dt, dev)
    _check("v", v, (B, Hkv, 2 * L, D), dt, dev)
    o = torch.empty_like(q) if out is None else out
    l_ = torch.empty((B, Hq, 2 * L), dtype=torch.float32, device=dev) if lse is None else lse
    _check("out", o, q.shape, dt, dev)
    _check("lse", l_, (B, Hq, 2 * L), torch.float32, dev)
    nbytes = _size(L, S)("bd_attn_workspace_bytes", B, L, S, Hq, Hkv, D, code, 0)
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    sh = _stream_handle(dev, stream)
    args = (_ptr(q), _ptr(k), _ptr(v), B, L, S, Hq, Hkv, D, _scale_arg(scale), code,
            _ptr(o), _ptr(l_), wp, wn, sh)
    if _marks:
        st = lib().bd_attn_fwd_marked(*args, *_marks_arg(_marks))
    else:
        st = lib().bd_attn_fwd(*args)
    if st:
        raise BdAttnError(st, "bd_attn_fwd")
    if stream is not None and workspace is None and ws is not None:
        ws.record_stream(stream)
    return o, l_


def bd_attn_bwd(do, q, k, v, o, lse, L: int, S: int, scale=None, dq=None, dk=None, dv=None,
                workspace=None, stream=None, _marks=None):
    """Backward pass; returns (dQ, dK, dV) in q's dtype."""
    B, Hq, Hkv, D = _shapes(q, k, L)
    dev, dt = q.device, q.dtype
    code = _dtype_code(q)
    for name, t, shp in (("do", do, q.shape), ("q", q, q.shape), ("k", k, (B, Hkv, 2 * L, D)),
                         ("v", v, (B, Hkv, 2 * L, D)), ("o", o, q.shape)):
        _check(name, t, shp, dt, dev)
    _check("lse", lse, (B, Hq, 2 * L), torch.float32, dev)
    dq_ = torch.empty_like(q) if dq is None else dq
    dk_ = torch.empty_like(k) if dk is None else dk
    dv_ = torch.empty_like(v) if dv is None else dv
    nbytes = _size(L, S)("bd_attn_workspace_bytes", B, L, S, Hq, Hkv, D, code, 1)
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    sh = _stream_handle(dev, stream)
    args = (_ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, L, S, Hq, Hkv, D,
            _scale_arg(scale), code, _ptr(dq_), _ptr(dk_), _ptr(dv_), wp, wn, sh)
    if _marks:
        st = lib().bd_attn_bwd_marked(*args, *_marks_arg(_marks))
    else:
        st = lib().bd_attn_bwd(*args)
    if st:
        raise BdAttnError(st, "bd_attn_bwd")
    if stream is not None and workspace is None and ws is not None:
        ws.record_stream(stream)
    return dq_, dk_, dv_


BD_ATTN_NOALLOC_SCRATCH_BYTES = 96 << 20   # the library's scratch array for bd_attn_bwd_noalloc


def bd_attn_bwd_noalloc(do, q, k, v, o, lse, L: int, S: int, dq, dk, dv, scale=None, stream=None):
    """bd_attn_bwd with the library's own scratch array as its workspace (for
    callers that cannot allocate): writes the caller's dq, dk, dv and returns
    them.  Calls whose work overlaps in time on one GPU race on that array."""
    B, Hq, Hkv, D = _shapes(q, k, L)
    dev, dt = q.device, q.dtype
    code = _dtype_code(q)
    for name, t, shp in (("do", do, q.shape), ("q", q, q.shape), ("k", k, (B, Hkv, 2 * L, D)),
                         ("v", v, (B, Hkv, 2 * L, D)), ("o", o, q.shape), ("dq", dq, q.shape),
                         ("dk", dk, (B, Hkv, 2 * L, D)), ("dv", dv, (B, Hkv, 2 * L, D))):
        _check(name, t, shp, dt, dev)
    _check("lse", lse, (B, Hq, 2 * L), torch.float32, dev)
    sh = _stream_handle(dev, stream)
    st = lib().bd_attn_bwd_noalloc(_ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, L, S, Hq, Hkv, D,
                                   _scale_arg(scale), code, _ptr(dq), _ptr(dk), _ptr(dv), sh)
    if st:
        raise BdAttnError(st, "bd_attn_bwd_noalloc")
    return dq, dk, dv


class BdAttnFunction(torch.autograd.Function):
    """Autograd wrapper: forward saves Q, K, V, O, LSE; backward returns dQ, dK, dV."""

    @staticmethod
    def forward(ctx, q, k, v, L, S, scale=None):
        o, lse = bd_attn_fwd(q, k, v, L, S, scale)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.L, ctx.S, ctx.scale = L, S, scale
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        dq, dk, dv = bd_attn_bwd(do.contiguous(), q, k, v, o, lse, ctx.L, ctx.S, ctx.scale)
        return dq, dk, dv, None, None, None


def bd_attn(q, k, v, L: int, S: int, scale=None):
    """Block-diffusion masked attention over [x_t | x_0]; differentiable."""
    return BdAttnFunction.apply(q, k, v, L, S, scale)


# ---------------------------------------------------------------------------
# Packed sequences: q [Hq, 2T, D], k/v [Hkv, 2T, D], cu_seqlens int32 [n+1] on
# the same device (cu_seqlens[0] = 0, cu_seqlens[n] = T); sequence i occupies
# rows [2 cu[i], 2 cu[i+1]) of every head, noisy copy first.

def bd_attn_varlen_workspace_bytes(n_seqs, total_L, max_L, S, Hq, Hkv, D, dtype, for_bwd) -> int:
    return int(lib().bd_attn_varlen_workspace_bytes(n_seqs, total_L, max_L, S, Hq, Hkv, D, int(dtype),
                                                      int(for_bwd)))


def _varlen_shapes(q, k, cu_seqlens):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q [Hq,2T,D] and k/v [Hkv,2T,D] expected")
    Hq, N, D = q.shape
    Hkv = k.shape[0]
    if N % 2:
        raise ValueError(f"packed length {N} is odd")
    if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
        raise ValueError("cu_seqlens must be a 1-D int32 tensor of n_seqs + 1 entries")
    if cu_seqlens.device != q.device or not cu_seqlens.is_contiguous():
        raise ValueError("cu_seqlens must be contiguous and on q's device")
    return Hq, Hkv, D, N // 2, cu_seqlens.numel() - 1


def bd_attn_varlen_fwd(q, k, v, cu_seqlens, max_L: int, S: int, scale=None, out=None, lse=None,
                       workspace=None, stream=None):
    """Forward pass over packed sequences; returns (O, LSE [Hq, 2T] float32)."""
    Hq, Hkv, D, T, n = _varlen_shapes(q, k, cu_seqlens)
    dev, dt = q.device, q.dtype
    code = _dtype_code(q)
    _check("k", k, (Hkv, 2 * T, D), dt, dev)
    _check("v", v, (Hkv, 2 * T, D), dt, dev)
    o = torch.empty_like(q) if out is None else out
    l_ = torch.empty((Hq, 2 * T), dtype=torch.float32, device=dev) if lse is None else lse
    _check("out", o, q.shape, dt, dev)
    _check("lse", l_, (Hq, 2 * T), torch.float32, dev)
    nbytes = _size(max_L, S)("bd_attn_varlen_workspace_bytes", n, T, max_L, S, Hq, Hkv, D, code, 0)
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    sh = _stream_handle(dev, stream)
    st = lib().bd_attn_varlen_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), n, T, max_L, S, Hq, Hkv, D,
                                  _scale_arg(scale), code, _ptr(o), _ptr(l_), wp, wn, sh)
    if st:
        raise BdAttnError(st, "bd_attn_varlen_fwd")
    if stream is not None and workspace is None and ws is not None:
        ws.record_stream(stream)
    return o, l_


def bd_attn_varlen_bwd(do, q, k, v, o, lse, cu_seqlens, max_L: int, S: int, scale=None, dq=None, dk=None,
                       dv=None, workspace=None, stream=None):
    """Backward pass over packed sequences; returns (dQ, dK, dV) in q's dtype."""
    Hq, Hkv, D, T, n = _varlen_shapes(q, k, cu_seqlens)
    dev, dt = q.device, q.dtype
    code = _dtype_code(q)
    for name, t, shp in (("do", do, q.shape), ("k", k, (Hkv, 2 * T, D)), ("v", v, (Hkv, 2 * T, D)),
                         ("o", o, q.shape)):
        _check(name, t, shp, dt, dev)
    _check("lse", lse, (Hq, 2 * T), torch.float32, dev)
    dq_ = torch.empty_like(q) if dq is None else dq
    dk_ = torch.empty_like(k) if dk is None else dk
    dv_ = torch.empty_like(v) if dv is None else dv
    nbytes = _size(max_L, S)("bd_attn_varlen_workspace_bytes", n, T, max_L, S, Hq, Hkv, D, code, 1)
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    sh = _stream_handle(dev, stream)
    st = lib().bd_attn_varlen_bwd(_ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(cu_seqlens), n,
                                  T, max_L, S, Hq, Hkv, D, _scale_arg(scale), code, _ptr(dq_), _ptr(dk_),
                                  _ptr(dv_), wp, wn, sh)
    if st:
        raise BdAttnError(st, "bd_attn_varlen_bwd")
    if stream is not None and workspace is None and ws is not None:
        ws.record_stream(stream)
    return dq_, dk_, dv_


class BdAttnVarlenFunction(torch.autograd.Function):
    """Autograd wrapper of the packed-sequence calls."""

    @staticmethod
    def forward(ctx, q, k, v, cu_seqlens, max_L, S, scale=None):
        o, lse = bd_attn_varlen_fwd(q, k, v, cu_seqlens, max_L, S, scale)
        ctx.save_for_backward(q, k, v, o, lse, cu_seqlens)
        ctx.max_L, ctx.S, ctx.scale = max_L, S, scale
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse, cu = ctx.saved_tensors
        dq, dk, dv = bd_attn_varlen_bwd(do.contiguous(), q, k, v, o, lse, cu, ctx.max_L, ctx.S, ctx.scale)
        return dq, dk, dv, None, None, None, None


def bd_attn_varlen(q, k, v, cu_seqlens, max_L: int, S: int, scale=None):
    """Block-diffusion masked attention over packed [x_t | x_0] sequences; differentiable."""
    return BdAttnVarlenFunction.apply(q, k, v, cu_seqlens, max_L, S, scale)


def bd_attn_decode_workspace_bytes(B, S, Hq, Hkv, D, capacity, dtype=BD_ATTN_BF16) -> int:
    return int(lib().bd_attn_decode_workspace_bytes(B, S, Hq, Hkv, D, capacity, int(dtype)))


def bd_attn_decode_fwd(q, k_cache, v_cache, k_new, v_new, cache_lens, scale=None, out=None, lse=None,
                       workspace=None, stream=None):
    """One block's decoding step over a KV cache; returns (O [B,Hq,S,D], LSE [B,Hq,S] float32).

    q [B,Hq,S,D]; k_cache/v_cache [B,Hkv,C,D]; k_new/v_new [B,Hkv,S,D], all
    bfloat16; cache_lens: int32 [B] on the device (clamped to [0, C])."""
    if q.dim() != 4 or k_cache.dim() != 4:
        raise ValueError("q [B,Hq,S,D] and k_cache/v_cache [B,Hkv,C,D] expected")
    B, Hq, S, D = q.shape
    Hkv, C = k_cache.shape[1], k_cache.shape[2]
    dev = q.device
    if q.dtype != torch.bfloat16:
        raise TypeError(f"bd_attn_decode_fwd supports bfloat16 tensors, got {q.dtype}")
    for name, t, shp in (("k_cache", k_cache, (B, Hkv, C, D)), ("v_cache", v_cache, (B, Hkv, C, D)),
                         ("k_new", k_new, (B, Hkv, S, D)), ("v_new", v_new, (B, Hkv, S, D))):
        _check(name, t, shp, torch.bfloat16, dev)
    _check("cache_lens", cache_lens, (B,), torch.int32, dev)
    o = torch.empty_like(q) if out is None else out
    l_ = torch.empty((B, Hq, S), dtype=torch.float32, device=dev) if lse is None else lse
    _check("out", o, q.shape, torch.bfloat16, dev)
    _check("lse", l_, (B, Hq, S), torch.float32, dev)
    nbytes = _known_size("bd_attn_decode_workspace_bytes", B, S, Hq, Hkv, D, C, BD_ATTN_BF16)
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    sh = _stream_handle(dev, stream)
    st = lib().bd_attn_decode_fwd(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_new), _ptr(v_new),
                                  _ptr(cache_lens), B, S, Hq, Hkv, D, C, _scale_arg(scale), BD_ATTN_BF16,
                                  _ptr(o), _ptr(l_), wp, wn, sh)
    if st:
        raise BdAttnError(st, "bd_attn_decode_fwd")
    if stream is not None and workspace is None and ws is not None:
        ws.record_stream(stream)
    return o, l_


# ---------------------------------------------------------------------------
# Token log-probabilities through the LM head (Eq. 3 and Eq. 6-7 objectives).

BD_LCE_CE = 0
BD_LCE_DIPO = 1


def bd_lce_workspace_bytes(N, V, Dm, for_bwd, dtype=BD_ATTN_BF16) -> int:
    return int(lib().bd_lce_workspace_bytes(N, V, Dm, int(dtype), int(for_bwd)))


def _lce_shapes(h, w, targets):
    if h.dim() != 2 or w.dim() != 2 or h.shape[1] != w.shape[1]:
        raise ValueError("h [N, Dm] and w [V, Dm] expected")
    N, Dm = h.shape
    V = w.shape[0]
    dev = h.device
    _check("h", h, (N, Dm), torch.bfloat16, dev)
    _check("w", w, (V, Dm), torch.bfloat16, dev)
    _check("targets", targets, (N,), torch.int32, dev)
    return N, V, Dm, dev


def bd_lce_logits_bytes(N, V, Dm, dtype=BD_ATTN_BF16) -> int:
    return int(lib().bd_lce_logits_bytes(N, V, Dm, int(dtype)))


def bd_lce_fwd(h, w, targets, lse=None, logp=None, workspace=None, stream=None, logits=None):
    """Per-position LSE and log p(target) (float32 [N]) of logits h w^T.
    logits: optional float32 tensor of bd_lce_logits_bytes bytes that receives
    the logits for bd_lce_bwd."""
    N, V, Dm, dev = _lce_shapes(h, w, targets)
    if logits is not None and (logits.dtype != torch.float32 or logits.numel() * 4 < bd_lce_logits_bytes(N, V, Dm)
                               or not logits.is_contiguous() or logits.device != dev):
        raise ValueError("logits: a contiguous float32 buffer of bd_lce_logits_bytes bytes on the device expected")
    l_ = torch.empty(N, dtype=torch.float32, device=dev) if lse is None else lse
    lp = torch.empty(N, dtype=torch.float32, device=dev) if logp is None else logp
    _check("lse", l_, (N,), torch.float32, dev)
    _check("logp", lp, (N,), torch.float32, dev)
    nbytes = _known_size("bd_lce_workspace_bytes", N, V, Dm, BD_ATTN_BF16, 0)
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    sh = _stream_handle(dev, stream)
    kl = None if logits is None else _ptr(logits)
    st = lib().bd_lce_fwd(_ptr(h), _ptr(w), _ptr(targets), N, V, Dm, BD_ATTN_BF16, _ptr(l_), _ptr(lp), kl, wp, wn, sh)
    if st:
        raise BdAttnError(st, "bd_lce_fwd")
    if stream is not None and workspace is None and ws is not None:
        ws.record_stream(stream)
    return l_, lp


def bd_lce_bwd(h, w, targets, lse, dlogp, dh=None, dw=None, workspace=None, stream=None, logits=None):
    """dH [N, Dm] and dW [V, Dm] (bf16) for dLoss/dlogp = dlogp (logits: the
    buffer bd_lce_fwd filled, to skip recomputing them)."""
    N, V, Dm, dev = _lce_shapes(h, w, targets)
    if logits is not None and (logits.dtype != torch.float32 or logits.numel() * 4 < bd_lce_logits_bytes(N, V, Dm)
                               or not logits.is_contiguous() or logits.device != dev):
        raise ValueError("logits: a contiguous float32 buffer of bd_lce_logits_bytes bytes on the device expected")
    _check("lse", lse, (N,), torch.float32, dev)
    _check("dlogp", dlogp, (N,), torch.float32, dev)
    dh_ = torch.empty_like(h) if dh is None else dh
    dw_ = torch.empty_like(w) if dw is None else dw
    _check("dh", dh_, (N, Dm), torch.bfloat16, dev)
    _check("dw", dw_, (V, Dm), torch.bfloat16, dev)
    nbytes = _known_size("bd_lce_workspace_bytes", N, V, Dm, BD_ATTN_BF16, 1)
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    sh = _stream_handle(dev, stream)
    kl = None if logits is None else _ptr(logits)
    st = lib().bd_lce_bwd(_ptr(h), _ptr(w), _ptr(targets), _ptr(lse), _ptr(dlogp), kl, N, V, Dm, BD_ATTN_BF16,
                          _ptr(dh_), _ptr(dw_), wp, wn, sh)
    if st:
        raise BdAttnError(st, "bd_lce_bwd")
    if stream is not None and workspace is None and ws is not None:
        ws.record_stream(stream)
    return dh_, dw_


def bd_lce_objective(logp, weight, kind=BD_LCE_CE, logp_old=None, logp_ref=None, adv=None, eps=0.2, beta=0.0,
                     loss=None, dlogp=None, stream=None):
    """Per-position loss and dloss/dlogp (float32 [N]) of the masked CE (kind
    BD_LCE_CE) or the DiPO clipped surrogate with KL (kind BD_LCE_DIPO)."""
    N = logp.numel()
    dev = logp.device
    for name, t in (("logp", logp), ("weight", weight), ("logp_old", logp_old), ("logp_ref", logp_ref),
                    ("adv", adv)):
        if t is not None:
            _check(name, t, (N,), torch.float32, dev)
    lo = torch.empty(N, dtype=torch.float32, device=dev) if loss is None else loss
    dl = torch.empty(N, dtype=torch.float32, device=dev) if dlogp is None else dlogp
    opt = lambda t: None if t is None else _ptr(t)  # noqa: E731
    sh = _stream_handle(dev, stream)
    st = lib().bd_lce_objective(_ptr(logp), opt(logp_old), opt(logp_ref), opt(adv), _ptr(weight), N, int(kind),
                                float(eps), float(beta), _ptr(lo), _ptr(dl), sh)
    if st:
        raise BdAttnError(st, "bd_lce_objective")
    return lo, dl


class LceFunction(torch.autograd.Function):
    """log p(target) through the LM head; differentiable in h and w."""

    @staticmethod
    def forward(ctx, h, w, targets, keep_logits=False):
        N, V, Dm, dev = _lce_shapes(h, w, targets)
        logits = (torch.empty(bd_lce_logits_bytes(N, V, Dm) // 4, dtype=torch.float32, device=dev)
                  if keep_logits else None)
        lse, logp = bd_lce_fwd(h, w, targets, logits=logits)
        ctx.save_for_backward(h, w, targets, lse)
        ctx.logits = logits
        return logp

    @staticmethod
    def backward(ctx, dlogp):
        h, w, targets, lse = ctx.saved_tensors
        dh, dw = bd_lce_bwd(h, w, targets, lse, dlogp.contiguous().float(), logits=ctx.logits)
        ctx.logits = None
        return dh, dw, None, None


def lm_head_logprobs(h, w, targets, keep_logits=False):
    """Differentiable per-position log p(target) [N] float32 (targets outside
    [0, V): 0).  keep_logits trades N x V float32 of memory for the
    backward's recomputation of the logits."""
    return LceFunction.apply(h, w, targets, keep_logits)


# ---------------------------------------------------------------------------
# Norms of queries and keys with the rotary embedding, in front of the
# attention: projections [B, N, H, D] (or [N, H, D]) with any strides in,
# contiguous heads [B, H, N, D] ([H, N, D]) out.

def _launch_context(device: torch.device, stream):
    """Where a call allocates and launches: on the tensors' device, and on
    `stream`, whose pool its results and workspace then come from."""
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"stream: expected one of {device}, got one of {stream.device}")
        return torch.cuda.stream(stream)
    if device.type == "cuda" and device.index != torch.cuda.current_device():
        return torch.cuda.device(device)
    return _HERE


_HERE = contextlib.nullcontext()


def _fit(*sizes) -> bool:
    """Do these sizes reach the library, which takes them as C ints, as they are?"""
    return max(sizes) < 1 << 31 and min(sizes) >= -1 << 31


def _check_fit(*sizes):
    if not _fit(*sizes):
        raise ValueError(f"sizes of at most 32 bits expected, got {sizes}")


def _row_strides(name, shape, strides):
    """Element strides (batch, token, head) of rows [.., N, H, D] of D contiguous values."""
    if strides[-1] != 1 and 0 not in shape:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    # (a dimension of one has no stride of its own)
    st = [s if n > 1 else 0 for n, s in zip(shape[:-1], strides[:-1])]
    if any(s % 8 for s in st):
        raise ValueError(f"{name}: strides must be multiples of 8 elements, got {strides}")
    return st if len(st) == 3 else [0] + st


# What a call derives from shapes and strides alone (checked on the way, and
# looked up once per combination, as a size is): the dimensions, the stride
# array of the C call, the shapes of the results and the strides of contiguous
# gradients.
_RopeLayout = collections.namedtuple("_RopeLayout", "B N Hq Hkv D strides pos_stride q_shape k_shape dense")


@functools.lru_cache(maxsize=1024)
def _rope_layout(q_shape, q_strides, k_shape, k_strides, v_shape, v_strides, pos_shape):
    if len(q_shape) not in (3, 4) or len(k_shape) != len(q_shape):
        raise ValueError("q [B,N,Hq,D] and k/v [B,N,Hkv,D] (or without B) expected")
    lead = tuple(q_shape[:-3])
    N, Hq, D = q_shape[-3:]
    Hkv = k_shape[-2]
    rows = (("q", q_shape, q_strides, Hq), ("k", k_shape, k_strides, Hkv), ("v", v_shape, v_strides, Hkv))
    strides = []
    for name, shape, st, H in rows[:2 if v_shape is None else 3]:
        if tuple(shape) != lead + (N, H, D):
            raise ValueError(f"{name}: expected shape {lead + (N, H, D)}, got {tuple(shape)}")
        strides += _row_strides(name, shape, st)
    if tuple(pos_shape) not in ((N,), lead + (N,)):
        raise ValueError(f"positions: expected shape {lead + (N,)} or {(N,)}, got {tuple(pos_shape)}")
    _check_fit(*lead, N, Hq, Hkv, D)
    dense = [s for H in (Hq, Hkv, Hkv) for s in (N * H * D, H * D, D)]
    return _RopeLayout(lead[0] if lead else 1, N, Hq, Hkv, D, (ctypes.c_int64 * len(strides))(*strides),
                       N if len(pos_shape) == 2 else 0,
                       lead + (Hq, N, D), lead + (Hkv, N, D), (ctypes.c_int64 * 9)(*dense))


@functools.lru_cache(maxsize=1024)
def _qkv_layout(shape, strides, Hq, Hkv, D, pos_shape):
    """_rope_layout of a fused projection [.., N, (Hq + 2 Hkv) D], whose heads start at multiples of D."""
    if len(shape) not in (2, 3) or shape[-1] != (Hq + 2 * Hkv) * D:
        raise ValueError(f"qkv [B,N,(Hq + 2 Hkv) D] (or without B) expected, got {tuple(shape)} for {Hq}/{Hkv} heads of {D}")
    heads = lambda H: (tuple(shape[:-1]) + (H, D), tuple(strides[:-1]) + (D * strides[-1], strides[-1]))  # noqa: E731
    return _rope_layout(*heads(Hq), *heads(Hkv), *heads(Hkv), pos_shape)


def _rope_inputs(lay, x, others, q_weight, k_weight, rope, positions):
    """Checks what a layout does not hold (types and devices; x: one of the projections, others: the rest) and
    returns the C call's arguments from the weights to wdtype but for eps, in two parts around it."""
    dt, dev, wdt, D = x.dtype, x.device, q_weight.dtype, lay.D
    for t in others:
        if t.dtype is not dt or t.device != dev:
            raise (TypeError if t.dtype != dt else ValueError)(
                f"q, k, v: one type and device expected, got {dt} on {dev} and {t.dtype} on {t.device}")
    code = _dtype_code(x)
    if wdt is not dt and wdt is not torch.float32:
        raise TypeError(f"q_weight: expected {dt} or torch.float32, got {wdt}")
    _check("q_weight", q_weight, (D,), wdt, dev)
    _check("k_weight", k_weight, (D,), wdt, dev)
    if rope.dim() != 2:
        raise ValueError("rope [n, D] expected")
    n = rope.shape[0]
    _check("rope", rope, (n, D), torch.float32, dev)
    _check("positions", positions, positions.shape, torch.int32, dev)
    head = (_ptr(q_weight), _ptr(k_weight), _ptr(rope), n, _ptr(positions), lay.pos_stride)
    return head, (code, code if wdt is dt else BD_ATTN_FP32)


def bd_rope_table(n: int, D: int, theta: float = 1e6, inv_freq=None, device="cuda", out=None, stream=None):
    """Rotary table of positions 0..n-1: float32 [n, D], the cosines of p f_j, then the sines.

    f_j = theta^(-2j/D), or inv_freq (float64 [D/2] on the device) for scaled
    frequencies.  Angles are formed in float64."""
    if out is not None:
        device = out.device
    elif inv_freq is not None:
        device = inv_freq.device
    _check_fit(n, D)
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    with _launch_context(device, stream):
        if inv_freq is None:
            inv_freq = float(theta) ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=device) / D)
        _check("inv_freq", inv_freq, (D // 2,), torch.float64, device)
        t = torch.empty((n, D), dtype=torch.float32, device=device) if out is None else out
        _check("out", t, (n, D), torch.float32, device)
        st = lib().bd_rope_table(_ptr(inv_freq), n, D, _ptr(t), _stream_handle(device, stream))
    if st:
        raise BdAttnError(st, "bd_rope_table")
    return t


def _result(name, t, like, shape):
    """The caller's array for a result, checked, or a new one, of `like`'s type and device."""
    if t is None:
        return like.new_empty(*shape)  # (half the time of torch.empty with a type and a device)
    _check(name, t, shape, like.dtype, like.device)
    return t


def bd_qk_norm_rope_fwd(q, k, v, q_weight, k_weight, rope, positions, eps: float = 1e-6, q_out=None, k_out=None,
                        v_out=None, stream=None):
    """Heads normalised (q, k), rotated (q, k) and laid out (q, k, v) for the attention.

    q [B,N,Hq,D], k, v [B,N,Hkv,D] in bfloat16 or float32, any strides that
    are multiples of 8 with D contiguous (views of a fused projection; without
    B for packed sequences); q_weight, k_weight [D] in that type or float32;
    rope: bd_rope_table; positions: int32 [B,N] or [N].  Returns q [B,Hq,N,D],
    k, v [B,Hkv,N,D], contiguous."""
    lay = _rope_layout(q.shape, q.stride(), k.shape, k.stride(), v.shape, v.stride(), positions.shape)
    args = _rope_inputs(lay, q, (k, v), q_weight, k_weight, rope, positions)
    return _rope_fwd(lay, q, (_ptr(q), _ptr(k), _ptr(v)), args, eps, q_out, k_out, v_out, stream)


def _rope_fwd(lay, x, ptrs, args, eps, q_out=None, k_out=None, v_out=None, stream=None):
    B, N, Hq, Hkv, D, strides, _, q_shape, k_shape = lay[:9]
    dev = x.device
    with _launch_context(dev, stream):
        qo = _result("q_out", q_out, x, q_shape)
        ko = _result("k_out", k_out, x, k_shape)
        vo = _result("v_out", v_out, x, k_shape)
        st = lib().bd_qk_norm_rope_fwd(*ptrs, strides, *args[0], B, N, Hq, Hkv, D, eps, *args[1], _ptr(qo), _ptr(ko),
                                       _ptr(vo), _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_qk_norm_rope_fwd")
    return qo, ko, vo


def bd_qk_norm_rope_workspace_bytes(B, N, Hq, Hkv, D, dtype=BD_ATTN_BF16) -> int:
    return int(lib().bd_qk_norm_rope_workspace_bytes(B, N, Hq, Hkv, D, int(dtype))) if _fit(B, N, Hq, Hkv, D) else 0


def bd_qk_norm_rope_bwd(dq, dk, dv, q, k, q_weight, k_weight, rope, positions, eps: float = 1e-6, grad_q=None,
                        grad_k=None, grad_v=None, grad_q_weight=None, grad_k_weight=None, workspace=None, stream=None):
    """Gradients of bd_qk_norm_rope_fwd for those of its results, dq [B,Hq,N,D] and dk, dv
    [B,Hkv,N,D] (contiguous): returns those of q, k, v (new, or the given arrays with any non-overlapping
    strides) and of the weights."""
    lay = _rope_layout(q.shape, q.stride(), k.shape, k.stride(), None, None, positions.shape)
    args = _rope_inputs(lay, q, (k,), q_weight, k_weight, rope, positions)
    dev, dt = q.device, q.dtype
    with _launch_context(dev, stream):
        grads, strides = [], lay.dense
        for name, t, like in (("grad_q", grad_q, q), ("grad_k", grad_k, k), ("grad_v", grad_v, k)):
            if t is None:
                t = torch.empty_like(like, memory_format=torch.contiguous_format)
            elif t.shape != like.shape or t.dtype != dt or t.device != dev:
                raise ValueError(f"{name}: expected {dt} {tuple(like.shape)} on {dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
            else:
                strides = None
            grads.append(t)
        gq, gk, gv = grads
        if strides is None:
            strides = _rope_layout(gq.shape, gq.stride(), gk.shape, gk.stride(), gv.shape, gv.stride(), positions.shape).strides
        gqw = _result("grad_q_weight", grad_q_weight, q_weight, (lay.D,))
        gkw = _result("grad_k_weight", grad_k_weight, q_weight, (lay.D,))
        _rope_bwd(lay, (dq, dk, dv), (_ptr(q), _ptr(k)), args, eps, dt, dev, (_ptr(gq), _ptr(gk), _ptr(gv)),
                  strides, gqw, gkw, workspace, stream)
    return (*grads, gqw, gkw)


def _rope_bwd(lay, dy, ptrs, args, eps, dtype, dev, grad_ptrs, grad_strides, gqw, gkw, workspace=None, stream=None):
    B, N, Hq, Hkv, D, strides, _, q_shape, k_shape = lay[:9]
    dq, dk, dv = dy
    _check("dq", dq, q_shape, dtype, dev)
    _check("dk", dk, k_shape, dtype, dev)
    _check("dv", dv, k_shape, dtype, dev)
    nbytes = _known_size("bd_qk_norm_rope_workspace_bytes", B, N, Hq, Hkv, D, args[1][0])
    ws, wp, wn = _workspace(nbytes, dev, workspace)
    st = lib().bd_qk_norm_rope_bwd(_ptr(dq), _ptr(dk), _ptr(dv), *ptrs, strides, *args[0], B, N, Hq, Hkv, D, eps, *args[1],
                                   *grad_ptrs, grad_strides, _ptr(gqw), _ptr(gkw), wp, wn, _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_qk_norm_rope_bwd")


class QkNormRopeFunction(torch.autograd.Function):
    """Autograd wrapper over separate projections."""

    @staticmethod
    def forward(ctx, q, k, v, q_weight, k_weight, rope, positions, eps):
        ctx.save_for_backward(q, k, q_weight, k_weight, rope, positions)
        ctx.eps = eps
        return bd_qk_norm_rope_fwd(q, k, v, q_weight, k_weight, rope, positions, eps)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        q, k, *rest = ctx.saved_tensors
        grads = bd_qk_norm_rope_bwd(dq.contiguous(), dk.contiguous(), dv.contiguous(), q, k, *rest, ctx.eps)
        return (*grads, None, None, None)


class QkvNormRopeFunction(torch.autograd.Function):
    """Autograd wrapper over a fused projection, whose gradient is written as one array."""

    @staticmethod
    def forward(ctx, qkv, Hq, Hkv, q_weight, k_weight, rope, positions, eps):
        ctx.save_for_backward(qkv, q_weight, k_weight, rope, positions)
        Hq, Hkv = operator.index(Hq), operator.index(Hkv)  # (only plain integers are looked up and kept)
        ctx.heads, ctx.eps = (Hq, Hkv), eps
        D = q_weight.numel()
        lay = _qkv_layout(qkv.shape, qkv.stride(), Hq, Hkv, D, positions.shape)
        args = _rope_inputs(lay, qkv, (), q_weight, k_weight, rope, positions)
        return _rope_fwd(lay, qkv, QkvNormRopeFunction._parts(qkv, Hq, Hkv, D), args, eps)

    @staticmethod
    def _parts(qkv, Hq, Hkv, D):
        """Addresses of the first query, key and value head."""
        p, el = _ptr(qkv), qkv.element_size()
        return p, p + Hq * D * el, p + (Hq + Hkv) * D * el

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        qkv, q_weight, k_weight, rope, positions = ctx.saved_tensors
        Hq, Hkv = ctx.heads
        D = q_weight.numel()
        dev, dt = qkv.device, qkv.dtype
        lay = _qkv_layout(qkv.shape, qkv.stride(), Hq, Hkv, D, positions.shape)
        args = _rope_inputs(lay, qkv, (), q_weight, k_weight, rope, positions)
        with _launch_context(dev, None):
            grad = torch.empty_like(qkv, memory_format=torch.contiguous_format)
            gqw, gkw = torch.empty_like(q_weight), torch.empty_like(k_weight)
            strides = _qkv_layout(grad.shape, grad.stride(), Hq, Hkv, D, positions.shape).strides
            _rope_bwd(lay, (dq.contiguous(), dk.contiguous(), dv.contiguous()),
                      QkvNormRopeFunction._parts(qkv, Hq, Hkv, D)[:2], args, ctx.eps, dt, dev,
                      QkvNormRopeFunction._parts(grad, Hq, Hkv, D), strides, gqw, gkw)
        return grad, None, None, gqw, gkw, None, None, None


def qk_norm_rope(q, k, v, q_weight, k_weight, rope, positions, eps: float = 1e-6):
    """bd_qk_norm_rope_fwd, differentiable in q, k, v and the weights.

    (As with any autograd function, a forward and its backward are captured into
    one graph, with no eager graph of the same leaves alive: torch's accumulation
    into a leaf runs on the stream of the first graph that used it.)"""
    return QkNormRopeFunction.apply(q, k, v, q_weight, k_weight, rope, positions, eps)


def qkv_norm_rope(qkv, Hq: int, Hkv: int, q_weight, k_weight, rope, positions, eps: float = 1e-6):
    """The same on a fused projection qkv [B, N, (Hq + 2 Hkv) D] (queries, keys, values)."""
    return QkvNormRopeFunction.apply(qkv, Hq, Hkv, q_weight, k_weight, rope, positions, eps)


# ---------------------------------------------------------------------------
# Paged KV cache: k_pages, v_pages [pages, Hkv, page_size, D] bfloat16 with any
# equal strides (a cache kept token-major is passed as its permuted view).

@functools.lru_cache(maxsize=1024)
def _page_layout(k_shape, k_strides, v_shape, v_strides, Hkv, D):
    """Page arguments of the C calls: pages, page size and the strides (of page, head and row)."""
    if len(k_shape) != 4:
        raise ValueError("k_pages and v_pages [pages,Hkv,page_size,D] expected")
    n, P = k_shape[0], k_shape[2]
    for name, shape in (("k_pages", k_shape), ("v_pages", v_shape)):
        if tuple(shape) != (n, Hkv, P, D):
            raise ValueError(f"{name}: expected shape {(n, Hkv, P, D)}, got {tuple(shape)}")
    # (a dimension of one page or head has no stride of its own)
    st, sv = (tuple(s if m > 1 else 0 for m, s in zip(k_shape[:3], strides[:3])) for strides in (k_strides, v_strides))
    if st != sv or k_strides[3] != 1 or v_strides[3] != 1:
        raise ValueError("k_pages and v_pages: equal strides with the last dimension contiguous expected")
    _check_fit(n, P)
    if any(s % 8 for s in st):
        raise ValueError(f"k_pages: strides must be multiples of 8 elements, got {k_strides}")
    return (n, P) + st


def _pages(k_pages, v_pages, Hkv, D, device):
    lay = _page_layout(k_pages.shape, k_pages.stride(), v_pages.shape, v_pages.stride(), Hkv, D)
    bf16 = torch.bfloat16
    if k_pages.dtype is bf16 and v_pages.dtype is bf16 and k_pages.device == device and v_pages.device == device:
        return lay
    for name, t in (("k_pages", k_pages), ("v_pages", v_pages)):
        if t.dtype is not torch.bfloat16:
            raise TypeError(f"{name}: expected {torch.bfloat16}, got {t.dtype}")
        if t.device != device:
            raise ValueError(f"{name}: expected device {device}, got {t.device}")
    return lay


def _table_stride(page_table, B, device, name="page_table"):
    """Checks a page table [B, max_pages] (rows contiguous) and returns the distance of its rows."""
    if page_table.dim() != 2 or page_table.shape[0] != B:
        raise ValueError(f"{name}: expected shape ({B}, max_pages), got {tuple(page_table.shape)}")
    if page_table.dtype is not torch.int32:
        raise TypeError(f"{name}: expected {torch.int32}, got {page_table.dtype}")
    width, (rows, cols) = page_table.shape[1], page_table.stride()
    if width >= 1 << 31:
        _check_fit(width)
    if page_table.device != device or (cols != 1 and width > 1):
        raise ValueError(f"{name}: contiguous rows on {device} expected")
    return rows if B > 1 else width


def bd_qk_norm_rope_paged(q, k, v, q_weight, k_weight, rope, positions, slots, k_pages, v_pages, eps: float = 1e-6,
                          q_out=None, stream=None):
    """bd_qk_norm_rope_fwd for serving: returns the queries [B,Hq,N,D] and writes keys and values into
    the pages, token (b, n) at row slots[b, n] (int32 [B,N] of bd_paged_plan; outside the pages: not written)."""
    lay = _rope_layout(q.shape, q.stride(), k.shape, k.stride(), v.shape, v.stride(), positions.shape)
    B, N, Hq, Hkv, D, strides, _, q_shape = lay[:8]
    dev = q.device
    if q.dtype != torch.bfloat16:
        raise TypeError(f"bd_qk_norm_rope_paged supports bfloat16 tensors, got {q.dtype}")
    head, types = _rope_inputs(lay, q, (k, v), q_weight, k_weight, rope, positions)
    _check("slots", slots, q.shape[:-2], torch.int32, dev)
    pages = _pages(k_pages, v_pages, Hkv, D, dev)
    with _launch_context(dev, stream):
        o = _result("q_out", q_out, q, q_shape)
        st = lib().bd_qk_norm_rope_paged(_ptr(q), _ptr(k), _ptr(v), strides, *head, _ptr(slots), B, N, Hq, Hkv, D, eps,
                                         *types, _ptr(o), _ptr(k_pages), _ptr(v_pages), *pages, _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_qk_norm_rope_paged")
    return o


PagedPlan = collections.namedtuple("PagedPlan", "lens cu slots positions state")


def bd_paged_plan(cache_lens, new_lens, page_table, free_pages, free_head, num_pages: int, page_size: int, S=None,
                  total=None, lens=None, cu=None, slots=None, positions=None, state=None, stream=None):
    """Pages and slots for the next tokens of a batch, from lengths on the device.

    cache_lens, new_lens: int32 [B]; page_table: int32 [B, max_pages] (rows may
    be strided), updated in place; free_pages: int32 [n]; free_head: int32 [1].
    With S, slots and positions are [B, S] (up to S new tokens a sequence),
    else [total], packed (total: at least the sum of new_lens).  Returns
    PagedPlan(lens [B], cu [B+1], slots, positions, state [2]): state[0] is the
    new head of the free list, state[1] the tokens without a slot."""
    dev = cache_lens.device
    B = cache_lens.numel()
    _check("cache_lens", cache_lens, (B,), torch.int32, dev)
    _check("new_lens", new_lens, (B,), torch.int32, dev)
    table_stride = _table_stride(page_table, B, dev)
    if free_pages.dim() != 1:
        raise ValueError("free_pages: 1-D expected")
    _check("free_pages", free_pages, (free_pages.numel(),), torch.int32, dev)
    _check("free_head", free_head, (1,), torch.int32, dev)
    if S is None and total is None:
        raise ValueError("S (rows of S tokens a sequence) or total (packed tokens) expected")
    if S is not None and S < 1:
        raise ValueError(f"S: at least 1 expected, got {S}")
    S_, total_ = (0, int(total)) if S is None else (int(S), 0)
    _check_fit(S_, total_, num_pages, page_size, free_pages.shape[0])
    shape = (B, S_) if S_ else (total_,)
    with _launch_context(dev, stream):
        lens = _result("lens", lens, cache_lens, (B,))
        cu = _result("cu", cu, cache_lens, (B + 1,))
        slots = _result("slots", slots, cache_lens, shape)
        positions = _result("positions", positions, cache_lens, shape)
        state = _result("state", state, cache_lens, (2,))
        st = lib().bd_paged_plan(_ptr(cache_lens), _ptr(new_lens), _ptr(page_table), B, page_table.shape[1], table_stride,
                                 _ptr(free_pages), free_pages.shape[0], _ptr(free_head), num_pages, page_size, S_, total_,
                                 _ptr(lens), _ptr(cu), _ptr(slots), _ptr(positions), _ptr(state),
                                 _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_paged_plan")
    return PagedPlan(lens, cu, slots, positions, state)


def bd_attn_paged_decode_workspace_bytes(B, S, Hq, Hkv, D, page_size, max_pages, dtype=BD_ATTN_BF16) -> int:
    if not _fit(B, S, Hq, Hkv, D, page_size, max_pages):
        return 0
    return int(lib().bd_attn_paged_decode_workspace_bytes(B, S, Hq, Hkv, D, page_size, max_pages, int(dtype)))


def _paged_inputs(call, q, k_pages, v_pages, k_new, v_new):
    """Checks the arrays that the decode calls over pages share: (shape of q, KV heads, device, page arguments,
    addresses of the block's keys and values)."""
    if q.dim() != 4 or k_pages.dim() != 4:
        raise ValueError("q [B,Hq,S,D] and k_pages/v_pages [pages,Hkv,page_size,D] expected")
    B, Hq, S, D = shape = q.shape
    Hkv, dev, bf16 = k_pages.shape[1], q.device, torch.bfloat16
    if q.dtype is not bf16:
        raise TypeError(f"{call} supports bfloat16 tensors, got {q.dtype}")
    if not q.is_contiguous():
        raise ValueError("q: must be contiguous")
    pages = _pages(k_pages, v_pages, Hkv, D, dev)
    if (k_new is None) != (v_new is None):
        raise ValueError("k_new and v_new: both or neither expected")
    kn = vn = None
    if k_new is not None:
        _check("k_new", k_new, (B, Hkv, S, D), bf16, dev)
        _check("v_new", v_new, (B, Hkv, S, D), bf16, dev)
        kn, vn = _ptr(k_new), _ptr(v_new)
    return shape, Hkv, dev, pages, kn, vn


def _paged_lse(lse, B, Hq, S, device):
    if lse is None:
        return torch.empty((B, Hq, S), dtype=torch.float32, device=device)
    _check("lse", lse, (B, Hq, S), torch.float32, device)
    return lse


def bd_attn_paged_decode_fwd(q, k_pages, v_pages, page_table, cache_lens, k_new=None, v_new=None, scale=None, out=None,
                             lse=None, workspace=None, stream=None):
    """bd_attn_decode_fwd over a paged cache; returns (O [B,Hq,S,D], LSE [B,Hq,S] float32).

    q [B,Hq,S,D] (S = 1: the next token of each sequence); k_pages, v_pages
    [pages,Hkv,page_size,D]; page_table int32 [B,max_pages] (rows may be
    strided); cache_lens int32 [B], clamped to [0, max_pages * page_size];
    k_new, v_new [B,Hkv,S,D]: the block's own keys, or None where the queries
    see the cache alone.  Rows that see no key: O = 0, LSE = -inf."""
    shape, Hkv, dev, (n, P, sp, sh, sr), kn, vn = _paged_inputs("bd_attn_paged_decode_fwd", q, k_pages, v_pages, k_new, v_new)
    B, Hq, S, D = shape
    table_stride = _table_stride(page_table, B, dev)
    width = page_table.shape[1]
    _check("cache_lens", cache_lens, (B,), torch.int32, dev)
    with _launch_context(dev, stream):
        o, l_ = _result("out", out, q, shape), _paged_lse(lse, B, Hq, S, dev)
        nbytes = _known_size("bd_attn_paged_decode_workspace_bytes", B, S, Hq, Hkv, D, P, width, BD_ATTN_BF16)
        ws, wp, wn = _workspace(nbytes, dev, workspace)
        st = lib().bd_attn_paged_decode_fwd(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(page_table), _ptr(cache_lens), kn,
                                            vn, B, S, Hq, Hkv, D, n, P, width, table_stride, sp, sh, sr, _scale_arg(scale),
                                            BD_ATTN_BF16, _ptr(o), _ptr(l_), wp, wn, _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_attn_paged_decode_fwd")
    return o, l_


def bd_attn_paged_shared_decode_workspace_bytes(B, groups, S, Hq, Hkv, D, page_size, max_prefix_pages, max_pages,
                                                dtype=BD_ATTN_BF16) -> int:
    if not _fit(B, groups, S, Hq, Hkv, D, page_size, max_prefix_pages, max_pages):
        return 0
    return int(lib().bd_attn_paged_shared_decode_workspace_bytes(B, groups, S, Hq, Hkv, D, page_size, max_prefix_pages,
                                                                 max_pages, int(dtype)))


def bd_attn_paged_shared_decode_fwd(q, k_pages, v_pages, group_sizes, prefix_table, prefix_lens, page_table, cache_lens,
                                    k_new=None, v_new=None, scale=None, out=None, lse=None, workspace=None, stream=None):
    """bd_attn_paged_decode_fwd for consecutive sequences that share a prefix, read once for the group.

    group_sizes int32 [groups]: sequences of each group, in order (sequences
    behind the last group have no prefix); prefix_table int32 [groups,
    max_prefix_pages] (rows may be strided) and prefix_lens int32 [groups]: the
    pages and keys of the prefixes; page_table, cache_lens and all else: the
    sequences' own keys, behind the prefix, as for bd_attn_paged_decode_fwd.
    (Empty groups and a prefix_table far wider than the prefixes cost time.)"""
    shape, Hkv, dev, (n, P, sp, sh, sr), kn, vn = _paged_inputs("bd_attn_paged_shared_decode_fwd", q, k_pages, v_pages, k_new, v_new)
    B, Hq, S, D = shape
    if group_sizes.dim() != 1:
        raise ValueError("group_sizes: 1-D expected")
    groups = group_sizes.shape[0]
    _check_fit(groups)
    _check("group_sizes", group_sizes, (groups,), torch.int32, dev)
    prefix_stride = _table_stride(prefix_table, groups, dev, "prefix_table")
    _check("prefix_lens", prefix_lens, (groups,), torch.int32, dev)
    table_stride = _table_stride(page_table, B, dev)
    prefix_width, width = prefix_table.shape[1], page_table.shape[1]
    _check("cache_lens", cache_lens, (B,), torch.int32, dev)
    with _launch_context(dev, stream):
        o, l_ = _result("out", out, q, shape), _paged_lse(lse, B, Hq, S, dev)
        nbytes = _known_size("bd_attn_paged_shared_decode_workspace_bytes", B, groups, S, Hq, Hkv, D, P, prefix_width, width,
                             BD_ATTN_BF16)
        ws, wp, wn = _workspace(nbytes, dev, workspace)
        st = lib().bd_attn_paged_shared_decode_fwd(
            _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(group_sizes), groups, _ptr(prefix_table), prefix_width,
            prefix_stride, _ptr(prefix_lens), _ptr(page_table), _ptr(cache_lens), kn, vn, B, S, Hq, Hkv, D, n, P, width,
            table_stride, sp, sh, sr, _scale_arg(scale), BD_ATTN_BF16, _ptr(o), _ptr(l_), wp, wn,
            _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_attn_paged_shared_decode_fwd")
    return o, l_


# ---------------------------------------------------------------------------
# Attention over chosen pages: summaries [pages, Hkv, 2, D] bfloat16 (smallest and
# largest keys of each page), lists of pages for each sequence and KV head.

def bd_paged_summarize(k_pages, page_table, from_lens, cache_lens, summaries, stream=None):
    """Updates the summaries of the pages that hold positions from_lens[b] up to cache_lens[b] (int32 [B]).

    k_pages [pages,Hkv,page_size,D] (any strides as for the other paged calls),
    page_table int32 [B,max_pages]; summaries [pages,Hkv,2,D] bfloat16, updated
    in place (the other pages' are left as they are, all of a sequence's where
    from_lens[b] >= cache_lens[b]) and returned."""
    if k_pages.dim() != 4:
        raise ValueError("k_pages [pages,Hkv,page_size,D] expected")
    Hkv, D, dev = k_pages.shape[1], k_pages.shape[3], k_pages.device
    n, P, sp, sh, sr = _pages(k_pages, k_pages, Hkv, D, dev)
    _check_fit(Hkv, D)
    B = cache_lens.numel()
    _check("from_lens", from_lens, (B,), torch.int32, dev)
    _check("cache_lens", cache_lens, (B,), torch.int32, dev)
    table_stride = _table_stride(page_table, B, dev)
    _check("summaries", summaries, (n, Hkv, 2, D), torch.bfloat16, dev)
    with _launch_context(dev, stream):
        st = lib().bd_paged_summarize(_ptr(k_pages), _ptr(page_table), _ptr(from_lens), _ptr(cache_lens), B, Hkv, D, n, P,
                                      page_table.shape[1], table_stride, sp, sh, sr, BD_ATTN_BF16, _ptr(summaries),
                                      _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_paged_summarize")
    return summaries


PagedLists = collections.namedtuple("PagedLists", "lists lens")


def bd_paged_select_workspace_bytes(B, S, Hq, Hkv, D, page_size, max_pages, budget, dtype=BD_ATTN_BF16) -> int:
    if not _fit(B, S, Hq, Hkv, D, page_size, max_pages, budget):
        return 0
    return int(lib().bd_paged_select_workspace_bytes(B, S, Hq, Hkv, D, page_size, max_pages, budget, int(dtype)))


def bd_paged_select(q, summaries, page_table, cache_lens, page_size: int, budget: int, first: int = 1, last: int = 1,
                    lists=None, lens=None, workspace=None, stream=None):
    """The pages that the queries of each sequence and KV head should attend to: the `first` first and `last`
    last of the sequence and those of the highest scores, `budget` in all (bounds of q . k by the summaries).

    q [B,Hq,S,D]; summaries [pages,Hkv,2,D] (bd_paged_summarize); page_table
    int32 [B,max_pages], cache_lens int32 [B].  Returns PagedLists(lists
    [B,Hkv,budget] in the order of positions, -1 behind them; lens [B,Hkv], the
    keys in them) for bd_attn_paged_sparse_decode_fwd."""
    if q.dim() != 4 or summaries.dim() != 4:
        raise ValueError("q [B,Hq,S,D] and summaries [pages,Hkv,2,D] expected")
    B, Hq, S, D = q.shape
    n, Hkv, dev, bf16 = summaries.shape[0], summaries.shape[1], q.device, torch.bfloat16
    _check("q", q, (B, Hq, S, D), bf16, dev)
    _check("summaries", summaries, (n, Hkv, 2, D), bf16, dev)
    page_size, budget, first, last = (operator.index(x) for x in (page_size, budget, first, last))
    table_stride = _table_stride(page_table, B, dev)
    width = page_table.shape[1]
    _check("cache_lens", cache_lens, (B,), torch.int32, dev)
    _check_fit(B, Hq, S, D, n, page_size, budget, first, last)
    if budget < 1:
        raise ValueError(f"budget: at least 1 expected, got {budget}")
    with _launch_context(dev, stream):
        lists = _result("lists", lists, cache_lens, (B, Hkv, budget))
        lens = _result("lens", lens, cache_lens, (B, Hkv))
        nbytes = _known_size("bd_paged_select_workspace_bytes", B, S, Hq, Hkv, D, page_size, width, budget, BD_ATTN_BF16)
        ws, wp, wn = _workspace(nbytes, dev, workspace)
        st = lib().bd_paged_select(_ptr(q), _ptr(summaries), _ptr(page_table), _ptr(cache_lens), B, S, Hq, Hkv, D, n,
                                   page_size, width, table_stride, budget, first, last, BD_ATTN_BF16, _ptr(lists), _ptr(lens),
                                   wp, wn, _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_paged_select")
    return PagedLists(lists, lens)


def bd_attn_paged_sparse_decode_workspace_bytes(B, S, Hq, Hkv, D, page_size, max_pages, dtype=BD_ATTN_BF16) -> int:
    if not _fit(B, S, Hq, Hkv, D, page_size, max_pages):
        return 0
    return int(lib().bd_attn_paged_sparse_decode_workspace_bytes(B, S, Hq, Hkv, D, page_size, max_pages, int(dtype)))


def bd_attn_paged_sparse_decode_fwd(q, k_pages, v_pages, lists, list_lens, k_new=None, v_new=None, scale=None, out=None,
                                    lse=None, workspace=None, stream=None):
    """bd_attn_paged_decode_fwd with pages of its own for each KV head: lists int32 [B,Hkv,max_pages]
    (contiguous), of which the first list_lens int32 [B,Hkv] keys are seen (bd_paged_select)."""
    shape, Hkv, dev, (n, P, sp, sh, sr), kn, vn = _paged_inputs("bd_attn_paged_sparse_decode_fwd", q, k_pages, v_pages, k_new, v_new)
    B, Hq, S, D = shape
    if lists.dim() != 3:
        raise ValueError("lists [B,Hkv,max_pages] expected")
    width = lists.shape[2]
    _check_fit(width)
    _check("lists", lists, (B, Hkv, width), torch.int32, dev)
    _check("list_lens", list_lens, (B, Hkv), torch.int32, dev)
    with _launch_context(dev, stream):
        o, l_ = _result("out", out, q, shape), _paged_lse(lse, B, Hq, S, dev)
        nbytes = _known_size("bd_attn_paged_sparse_decode_workspace_bytes", B, S, Hq, Hkv, D, P, width, BD_ATTN_BF16)
        ws, wp, wn = _workspace(nbytes, dev, workspace)
        st = lib().bd_attn_paged_sparse_decode_fwd(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(lists), _ptr(list_lens), kn,
                                                   vn, B, S, Hq, Hkv, D, n, P, width, sp, sh, sr, _scale_arg(scale),
                                                   BD_ATTN_BF16, _ptr(o), _ptr(l_), wp, wn, _stream_handle(dev, stream))
    if st:
        raise BdAttnError(st, "bd_attn_paged_sparse_decode_fwd")
    return o, l_
