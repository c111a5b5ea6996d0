"""Python binding of libkvs (ctypes).  Argument marshalling only.

The functions named ``kvs_*`` mirror the C ABI in ``include/kvs.h`` one to
one, taking torch tensors in place of device pointers and passing the
current HIP stream.  ``evict_attn`` wraps forward and backward in a
``torch.autograd.Function``.  torch provides device memory and streams
only; every step of the computation runs in the library's HIP kernels.

Importing this module fails if ``libkvs.so`` has not been built.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
from typing import Optional, Tuple

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkvs.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2609_35750_amd.build` (needs hipcc)")

lib = ctypes.CDLL(LIB_PATH)

_P, _I, _F, _Z, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_int64

SIGNATURES = {
    "kvs_abi_version": (_I, []),
    "kvs_status_string": (ctypes.c_char_p, [_I]),
    "kvs_last_error": (ctypes.c_char_p, []),
    "kvs_evict_attn_fwd_workspace": (_Z, [_I, _I, _I, _I, _I]),
    "kvs_evict_attn_fwd": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _P, _Z, _P]),
    "kvs_evict_attn_bwd_workspace": (_Z, [_I, _I, _I, _I, _I]),
    "kvs_evict_attn_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _P, _Z, _P]),
    "kvs_evict_attn_varlen_fwd_workspace": (_Z, [_I, _I, _I, _I, _I, _I]),
    "kvs_evict_attn_varlen_fwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P, _Z, _P]),
    "kvs_evict_attn_varlen_bwd_workspace": (_Z, [_I, _I, _I, _I, _I, _I]),
    "kvs_evict_attn_varlen_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                       _I, _I, _I, _I, _I, _I, _F, _P, _Z, _P]),
    "kvs_evict_attn_fwd_ex": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, ctypes.c_uint,
                                   _P, _Z, _P]),
    "kvs_evict_attn_bwd_ex": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                   _I, _I, _I, _I, _I, _I, _F, ctypes.c_uint, _P, _Z, _P]),
    "kvs_evict_attn_fwd_noalloc": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P]),
    "kvs_window_attn_fwd_workspace": (_Z, [_I, _I, _I, _I, _I, _I]),
    "kvs_window_attn_fwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _I, _I, _P, _Z, _P]),
    "kvs_window_attn_bwd_workspace": (_Z, [_I, _I, _I, _I, _I, _I]),
    "kvs_window_attn_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                 _I, _I, _I, _I, _I, _I, _F, _I, _I, _P, _Z, _P]),
    "kvs_window_attn_fwd_rem": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _I, _I, _P, _Z, _P]),
    "kvs_window_attn_bwd_rem": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                     _I, _I, _I, _I, _I, _I, _F, _I, _I, _P, _Z, _P]),
    "kvs_key_weights_workspace": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "kvs_key_weights": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _I, _I, _I, _P, _Z, _P]),
    "kvs_classify_tiles": (_I, [_P, _P, _I, _I, _I, _I, _P, _P]),
    "kvs_classify_tiles_size": (_Z, [ctypes.POINTER(ctypes.c_int32), _I, _I, _I]),
    "kvs_check_evict_at": (_I, [_P, _P, _I, _I, ctypes.POINTER(_L), _P]),
    "kvs_prof_enable": (None, [_I]),
    "kvs_prof_reset": (None, []),
    "kvs_prof_read": (_I, [ctypes.c_char_p, ctypes.POINTER(_I), ctypes.POINTER(ctypes.c_double)]),
    # streamed paged KV cache (host block manager: host int32 arrays)
    "kvs_bm_create": (_I, [_I, _I, _I, _I, ctypes.POINTER(_P)]),
    "kvs_bm_destroy": (None, [_P]),
    "kvs_bm_append": (_I, [_P, _I, _P, _I, _P]),
    "kvs_bm_evict": (_I, [_P, _I, _P, _I, _P]),
    "kvs_bm_release": (_I, [_P, _I, _P, ctypes.POINTER(_I)]),
    "kvs_bm_tables": (_I, [_P, _P, _P]),
    "kvs_bm_free_blocks": (_I, [_P]),
    "kvs_bm_live": (_I, [_P, _I]),
    "kvs_bm_fork": (_I, [_P, _I, _I]),
    "kvs_bm_evict_shared": (_I, [_P, _I, _P, _I, _P, _P, _P, ctypes.POINTER(_I)]),
    "kvs_bm_copy": (_I, [_P, _I, _I, _P, _P, ctypes.POINTER(_I)]),
    "kvs_bm_compact": (_I, [_P, _I, _P, _P, ctypes.POINTER(_I)]),
    "kvs_bm_groups": (_I, [_P, _P, _P, ctypes.POINTER(_I)]),
    "kvs_bm_shared": (_I, [_P, _I]),
    "kvs_paged_append": (_I, [_P, _P, _P, _P, _I, _P, _P, _P, _I, _I, _I, _I, _P]),
    "kvs_paged_evict": (_I, [_P, _I, _P, _I, _I, _P]),
    "kvs_paged_append_host": (_I, [_P, _P, _P, _P, _I, _P, _P, _P, _I, _I, _I, _I, _P]),
    "kvs_paged_evict_host": (_I, [_P, _I, _P, _I, _I, _P]),
    "kvs_paged_append_weighted": (_I, [_P, _P, _P, _P, _P, _I, _P, _P, _P, _P, _I, _I, _I, _I, _P]),
    "kvs_paged_append_weighted_host": (_I, [_P, _P, _P, _P, _P, _I, _P, _P, _P, _P, _I, _I, _I, _I, _P]),
    "kvs_paged_evict_lowest_workspace": (_Z, [_I, _I, _I]),
    "kvs_paged_evict_lowest": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _P, _Z, _P]),
    "kvs_paged_decode_ex_workspace": (_Z, [_I, _I, _I, _I, _I, _I, _I, _I, _I, _I]),
    "kvs_paged_decode_ex": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _F, _I, _I,
                                 _P, _Z, _P]),
    "kvs_paged_copy": (_I, [_P, _P, _I, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P]),
    "kvs_paged_decode_shared_workspace": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "kvs_paged_decode_shared": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _F, _P, _Z,
                                     _P]),
    "kvs_paged_extend_workspace": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "kvs_paged_extend": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _F, _I, _I, _P, _Z,
                              _P]),
    "kvs_paged_decode_workspace": (_Z, [_I, _I, _I, _I, _I, _I]),
    "kvs_paged_decode": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _F, _P, _Z, _P]),
}
for _name, (_res, _args) in SIGNATURES.items():
    _fn = getattr(lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

KVS_OK, KVS_ERR_NULL, KVS_ERR_SHAPE, KVS_ERR_ALIGN, KVS_ERR_WORKSPACE, KVS_ERR_EVICT, KVS_ERR_HIP, \
    KVS_ERR_UNSUPPORTED, KVS_ERR_CAPACITY, KVS_ERR_STATE = range(10)
# tile-classifier switches of the *_ex calls (consistency checks)
FLAG_NO_EMPTY_SKIP, FLAG_FULL_AS_PARTIAL = 1, 2


class KvsError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        msg = lib.kvs_status_string(status).decode()
        detail = lib.kvs_last_error().decode()
        super().__init__(f"{fn}: {msg}" + (f" ({detail})" if detail else ""))


def _check(fn: str, status: int) -> None:
    if status != KVS_OK:
        raise KvsError(fn, status)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


# The current stream's handle alone; no public name gives it, so a torch without this one makes the Stream object
# (2 us on every call's way to the GPU).
_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor):
    return torch.cuda.current_stream(t.device).cuda_stream if _RAW_STREAM is None else _RAW_STREAM(t.device.index)


def _workspace(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator returns blocks aligned to at least 512 bytes
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def _dims(q, k, cu_seqlens):
    if cu_seqlens is None:
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("fixed-length tensors are [B, T, H, D]")
        B, T, Hq, D = q.shape
        return B, T, B * T, Hq, k.shape[2], D
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("varlen tensors are [Ntot, H, D]")
    Ntot, Hq, D = q.shape
    return cu_seqlens.numel() - 1, None, Ntot, Hq, k.shape[1], D


def _check_dtypes(evict_at, cu_seqlens, *bf16):
    for t in bf16:
        if t.dtype != torch.bfloat16:
            raise ValueError("Q, K, V, O, dO must be bfloat16")
    if evict_at.dtype != torch.int32 or (cu_seqlens is not None and cu_seqlens.dtype != torch.int32):
        raise ValueError("evict_at and cu_seqlens must be int32")


def _check_shapes(q, k, v, evict_at, cu_seqlens, max_seqlen, check_cu, *like_q):
    """Host-side consistency of the tensor shapes (the library only sees pointers)."""
    if k.shape != v.shape or k.shape[:-2] != q.shape[:-2] or k.shape[-1] != q.shape[-1]:
        raise ValueError(f"shape mismatch: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    for t in like_q:
        if t.shape != q.shape:
            raise ValueError(f"shape mismatch: {tuple(t.shape)} vs q {tuple(q.shape)}")
    if evict_at.shape != q.shape[:-2]:
        raise ValueError(f"evict_at has shape {tuple(evict_at.shape)}, expected {tuple(q.shape[:-2])}")
    if cu_seqlens is not None and check_cu:
        cu = cu_seqlens.cpu().tolist()
        if cu[0] != 0 or cu[-1] != q.shape[0] or any(b < a for a, b in zip(cu[:-1], cu[1:])):
            raise ValueError("cu_seqlens must be 0 = cu[0] <= ... <= cu[B] = Ntot")
        if max(b - a for a, b in zip(cu[:-1], cu[1:])) > int(max_seqlen):
            raise ValueError("max_seqlen is smaller than a trace length")


def kvs_evict_attn_fwd(q, k, v, evict_at, softmax_scale=None, cu_seqlens=None, max_seqlen=None,
                       out=None, lse=None, check_cu=True, flags=0) -> Tuple[torch.Tensor, torch.Tensor]:
    """Forward of eviction-masked attention; returns ``(O, LSE)``.

    Fixed length: q [B,T,Hq,D], k/v [B,T,Hkv,D], evict_at [B,T] -> LSE [B,Hq,T].
    Varlen (``cu_seqlens`` int32 [B+1] on the GPU, ``max_seqlen`` int): q [Ntot,Hq,D],
    k/v [Ntot,Hkv,D], evict_at [Ntot] -> LSE [Hq,Ntot].
    Nonzero ``flags`` (FLAG_*) go through ``kvs_evict_attn_fwd_ex``.
    """
    _check_dtypes(evict_at, cu_seqlens, q, k, v)
    B, T, ntok, Hq, Hkv, D = _dims(q, k, cu_seqlens)
    scale = 1.0 / math.sqrt(D) if softmax_scale is None else float(softmax_scale)
    out = torch.empty_like(q) if out is None else out
    lse_shape = (B, Hq, T) if cu_seqlens is None else (Hq, ntok)
    if lse is None:
        lse = torch.empty(lse_shape, dtype=torch.float32, device=q.device)
    if tuple(lse.shape) != lse_shape or lse.dtype != torch.float32:
        raise ValueError(f"LSE must be float32 {lse_shape}")
    _check_shapes(q, k, v, evict_at, cu_seqlens, max_seqlen, check_cu, out)
    s = _stream(q)
    if flags:
        mx = T if cu_seqlens is None else max_seqlen
        if mx is None:
            raise ValueError("max_seqlen is required with cu_seqlens")
        nws = (lib.kvs_evict_attn_fwd_workspace(B, T, Hq, Hkv, D) if cu_seqlens is None else
               lib.kvs_evict_attn_varlen_fwd_workspace(B, ntok, int(mx), Hq, Hkv, D))
        ws = _workspace(nws, q.device)
        st = lib.kvs_evict_attn_fwd_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(evict_at), _ptr(cu_seqlens), _ptr(out),
                                       _ptr(lse), B, ntok, int(mx), Hq, Hkv, D, scale, int(flags), _ptr(ws), nws, s)
    elif cu_seqlens is None:
        nws = lib.kvs_evict_attn_fwd_workspace(B, T, Hq, Hkv, D)
        ws = _workspace(nws, q.device)
        st = lib.kvs_evict_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(evict_at), _ptr(out), _ptr(lse),
                                    B, T, Hq, Hkv, D, scale, _ptr(ws), nws, s)
    else:
        if max_seqlen is None:
            raise ValueError("max_seqlen is required with cu_seqlens")
        nws = lib.kvs_evict_attn_varlen_fwd_workspace(B, ntok, int(max_seqlen), Hq, Hkv, D)
        ws = _workspace(nws, q.device)
        st = lib.kvs_evict_attn_varlen_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(evict_at), _ptr(cu_seqlens),
                                           _ptr(out), _ptr(lse), B, ntok, int(max_seqlen), Hq, Hkv, D, scale,
                                           _ptr(ws), nws, s)
    _check("kvs_evict_attn_fwd", st)
    return out, lse


def kvs_evict_attn_bwd(do, q, k, v, o, lse, evict_at, softmax_scale=None, cu_seqlens=None, max_seqlen=None,
                       dq=None, dk=None, dv=None, check_cu=True,
                       flags=0) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Backward of eviction-masked attention; returns ``(dQ, dK, dV)`` (bf16).
    Nonzero ``flags`` (FLAG_*) go through ``kvs_evict_attn_bwd_ex``."""
    _check_dtypes(evict_at, cu_seqlens, q, k, v, o, do)
    B, T, ntok, Hq, Hkv, D = _dims(q, k, cu_seqlens)
    scale = 1.0 / math.sqrt(D) if softmax_scale is None else float(softmax_scale)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    lse_shape = (B, Hq, T) if cu_seqlens is None else (Hq, ntok)
    if tuple(lse.shape) != lse_shape or lse.dtype != torch.float32:
        raise ValueError(f"LSE must be float32 {lse_shape}")
    _check_shapes(q, k, v, evict_at, cu_seqlens, max_seqlen, check_cu, o, do, dq)
    if dk.shape != k.shape or dv.shape != k.shape:
        raise ValueError("dK, dV must have the shape of K")
    s = _stream(q)
    if flags:
        mx = T if cu_seqlens is None else max_seqlen
        if mx is None:
            raise ValueError("max_seqlen is required with cu_seqlens")
        nws = (lib.kvs_evict_attn_bwd_workspace(B, T, Hq, Hkv, D) if cu_seqlens is None else
               lib.kvs_evict_attn_varlen_bwd_workspace(B, ntok, int(mx), Hq, Hkv, D))
        ws = _workspace(nws, q.device)
        st = lib.kvs_evict_attn_bwd_ex(_ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(evict_at),
                                       _ptr(cu_seqlens), _ptr(dq), _ptr(dk), _ptr(dv), B, ntok, int(mx), Hq, Hkv, D,
                                       scale, int(flags), _ptr(ws), nws, s)
    elif cu_seqlens is None:
        nws = lib.kvs_evict_attn_bwd_workspace(B, T, Hq, Hkv, D)
        ws = _workspace(nws, q.device)
        st = lib.kvs_evict_attn_bwd(_ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(evict_at),
                                    _ptr(dq), _ptr(dk), _ptr(dv), B, T, Hq, Hkv, D, scale, _ptr(ws), nws, s)
    else:
        if max_seqlen is None:
            raise ValueError("max_seqlen is required with cu_seqlens")
        nws = lib.kvs_evict_attn_varlen_bwd_workspace(B, ntok, int(max_seqlen), Hq, Hkv, D)
        ws = _workspace(nws, q.device)
        st = lib.kvs_evict_attn_varlen_bwd(_ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                           _ptr(evict_at), _ptr(cu_seqlens), _ptr(dq), _ptr(dk), _ptr(dv),
                                           B, ntok, int(max_seqlen), Hq, Hkv, D, scale, _ptr(ws), nws, s)
    _check("kvs_evict_attn_bwd", st)
    return dq, dk, dv


_HERE = contextlib.nullcontext()


def _on(t: torch.Tensor):
    """Context in which t's device is the current one (nothing to do, the usual case, if it is)."""
    return _HERE if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)


def _i31(x) -> int:
    """A count as a C int: values beyond its range count as the largest (or as negative)."""
    return max(-1, min(int(x), 0x7FFFFFFF))


def _window_args(tensors, bf16, fp32, q, k, evict_at, cu_seqlens, max_seqlen, softmax_scale, check_cu):
    """Checks shared by the calls under a window; returns (B, Ntot, max_seqlen, Hq, Hkv, D, scale, LSE shape)."""
    for t in tensors:
        if t is not None and t.device != q.device:
            raise ValueError("tensors must be on one device")
    for t in bf16:
        if t.dtype != torch.bfloat16:
            raise ValueError("Q, K, V, O, dO and their gradients must be bfloat16")
    for t in fp32:
        if t.dtype != torch.float32:
            raise ValueError("LSE and W must be float32")
    for t in (evict_at, cu_seqlens):
        if t is not None and t.dtype != torch.int32:
            raise ValueError("evict_at and cu_seqlens must be int32")
    B, T, ntok, Hq, Hkv, D = _dims(q, k, cu_seqlens)
    if cu_seqlens is not None:
        if max_seqlen is None:
            raise ValueError("max_seqlen is required with cu_seqlens")
        T = _i31(max_seqlen)
    if k.shape[:-2] != q.shape[:-2] or k.shape[-1] != D:
        raise ValueError(f"shape mismatch: q {tuple(q.shape)}, k {tuple(k.shape)}")
    if evict_at is not None and evict_at.shape != q.shape[:-2]:
        raise ValueError(f"evict_at has shape {tuple(evict_at.shape)}, expected {tuple(q.shape[:-2])}")
    if cu_seqlens is not None and check_cu:
        _check_shapes(q, k, k, q[..., 0, 0], cu_seqlens, T, True)
    if not q.is_cuda:
        raise ValueError("tensors must be on the GPU")
    scale = 1.0 / math.sqrt(D) if softmax_scale is None else float(softmax_scale)
    return B, ntok, T, Hq, Hkv, D, scale, (B, Hq, T) if cu_seqlens is None else (Hq, ntok)


def _like(t, ref, name):
    if t.shape != ref.shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(ref.shape)}")


def _rem_like(rem, q):
    if rem is not None:
        if rem.dtype != torch.int8:
            raise ValueError("the remainders of O must be int8")
        _like(rem, q, "the remainders of O")


def kvs_window_attn_fwd(q, k, v, window: int, sinks: int = 0, evict_at=None, softmax_scale=None, cu_seqlens=None,
                        max_seqlen=None, out=None, lse=None, check_cu=True,
                        rem=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Forward of attention under a sliding window with sinks; returns ``(O, LSE)``.

    Query i sees key j iff ``j <= i``, ``i < evict_at[j]`` (if given) and ``i - j < window or j < sinks``.
    Layouts as in ``kvs_evict_attn_fwd``; ``check_cu=False`` skips the host's look at ``cu_seqlens`` (a
    synchronisation, which a stream that is being captured does not take).  ``rem`` (int8, O's shape) receives what
    O's rounding takes, for a backward whose Delta is that of the unrounded O.
    """
    out = torch.empty_like(q) if out is None else out
    B, n, T, Hq, Hkv, D, scale, lse_shape = _window_args((k, v, evict_at, cu_seqlens, out, lse, rem), (q, k, v, out), (), q,
                                                         k, evict_at, cu_seqlens, max_seqlen, softmax_scale, check_cu)
    if lse is None:
        lse = torch.empty(lse_shape, dtype=torch.float32, device=q.device)
    if tuple(lse.shape) != lse_shape or lse.dtype != torch.float32:
        raise ValueError(f"LSE must be float32 {lse_shape}")
    _like(v, k, "V")
    _like(out, q, "O")
    _rem_like(rem, q)
    nws = lib.kvs_window_attn_fwd_workspace(B, n, T, Hq, Hkv, D)
    ws = _workspace(nws, q.device)
    with _on(q):
        st = lib.kvs_window_attn_fwd_rem(_ptr(q), _ptr(k), _ptr(v), _ptr(evict_at), _ptr(cu_seqlens), _ptr(out), _ptr(rem),
                                         _ptr(lse), B, n, T, Hq, Hkv, D, scale, _i31(window), _i31(sinks), _ptr(ws), nws,
                                         _stream(q))
    _check("kvs_window_attn_fwd", st)
    return out, lse


def kvs_window_attn_bwd(do, q, k, v, o, lse, window: int, sinks: int = 0, evict_at=None, softmax_scale=None,
                        cu_seqlens=None, max_seqlen=None, dq=None, dk=None, dv=None, check_cu=True,
                        rem=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Backward of ``kvs_window_attn_fwd``; returns ``(dQ, dK, dV)`` (bf16).  ``rem``: the forward's."""
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    B, n, T, Hq, Hkv, D, scale, lse_shape = _window_args((do, k, v, o, lse, evict_at, cu_seqlens, dq, dk, dv, rem),
                                                         (do, q, k, v, o, dq, dk, dv), (lse,), q, k, evict_at,
                                                         cu_seqlens, max_seqlen, softmax_scale, check_cu)
    if tuple(lse.shape) != lse_shape:
        raise ValueError(f"LSE must be float32 {lse_shape}")
    for t, ref, name in ((do, q, "dO"), (o, q, "O"), (dq, q, "dQ"), (v, k, "V"), (dk, k, "dK"), (dv, k, "dV")):
        _like(t, ref, name)
    _rem_like(rem, q)
    nws = lib.kvs_window_attn_bwd_workspace(B, n, T, Hq, Hkv, D)
    ws = _workspace(nws, q.device)
    with _on(q):
        st = lib.kvs_window_attn_bwd_rem(_ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(rem), _ptr(lse),
                                         _ptr(evict_at), _ptr(cu_seqlens), _ptr(dq), _ptr(dk), _ptr(dv), B, n, T, Hq, Hkv,
                                         D, scale, _i31(window), _i31(sinks), _ptr(ws), nws, _stream(q))
    _check("kvs_window_attn_bwd", st)
    return dq, dk, dv


def kvs_key_weights(q, k, lse, evict_at=None, softmax_scale=None, cu_seqlens=None, max_seqlen=None,
                    window: Optional[int] = None, sinks: int = 0, last_rows: Optional[int] = None, out=None,
                    check_cu=True) -> torch.Tensor:
    """Attention weight of every key, ``W_j = sum over heads and over the queries i that see j of exp(s_ij - LSE_i)``.

    ``lse`` is the forward's over the same mask (``window`` None: no window).  ``last_rows`` (None: all) counts the
    last queries of each trace only.  Returns float32 [B, T] (varlen: [Ntot]).
    """
    if window is not None and window < 1:
        raise ValueError("window must be >= 1 (None: no window)")
    if last_rows is not None and last_rows < 1:
        raise ValueError("last_rows must be >= 1 (None: all)")
    w = torch.empty(q.shape[:-2], dtype=torch.float32, device=q.device) if out is None else out
    B, n, T, Hq, Hkv, D, scale, lse_shape = _window_args((k, lse, evict_at, cu_seqlens, w), (q, k), (lse, w), q, k,
                                                         evict_at, cu_seqlens, max_seqlen, softmax_scale, check_cu)
    if tuple(lse.shape) != lse_shape:
        raise ValueError(f"LSE must be float32 {lse_shape}")
    if w.shape != q.shape[:-2]:
        raise ValueError(f"W has shape {tuple(w.shape)}, expected {tuple(q.shape[:-2])}")
    rows = 0 if last_rows is None else _i31(last_rows)
    nws = lib.kvs_key_weights_workspace(B, n, T, Hq, Hkv, D, rows)
    ws = _workspace(nws, q.device)
    with _on(q):
        st = lib.kvs_key_weights(_ptr(q), _ptr(k), _ptr(lse), _ptr(evict_at), _ptr(cu_seqlens), _ptr(w), B, n, T, Hq,
                                 Hkv, D, scale, _i31(window or 0), _i31(sinks), rows, _ptr(ws), nws, _stream(q))
    _check("kvs_key_weights", st)
    return w


def kvs_classify_tiles(evict_at, BM: int, BN: int, cu_seqlens=None) -> torch.Tensor:
    """Tile classes (uint8: 0 EMPTY, 1 PARTIAL, 2 FULL), per-trace grids concatenated.

    ``evict_at`` is [B, T] (or [T]) without ``cu_seqlens``, else packed [Ntot]."""
    if evict_at.dtype != torch.int32:
        raise ValueError("evict_at must be int32")
    if cu_seqlens is None:
        B, T = evict_at.shape if evict_at.dim() == 2 else (1, evict_at.numel())
        lens = [T] * B
    else:
        B, T = cu_seqlens.numel() - 1, evict_at.numel()
        lens = (cu_seqlens[1:] - cu_seqlens[:-1]).cpu().tolist()   # sizes the output buffer
    arr = (ctypes.c_int32 * B)(*lens)
    n = lib.kvs_classify_tiles_size(arr, B, BM, BN)
    out = torch.empty(max(n, 1), dtype=torch.uint8, device=evict_at.device)
    st = lib.kvs_classify_tiles(_ptr(evict_at), _ptr(cu_seqlens), B, T, BM, BN, _ptr(out), _stream(evict_at))
    _check("kvs_classify_tiles", st)
    return out[:n]


def kvs_check_evict_at(evict_at, cu_seqlens=None) -> int:
    """Returns -1 if every evict_at[j] > j (trace-local), else the first bad packed index."""
    if cu_seqlens is None:
        B, T = evict_at.shape if evict_at.dim() == 2 else (1, evict_at.numel())
    else:
        B, T = cu_seqlens.numel() - 1, evict_at.numel()
    fb = ctypes.c_int64(-1)
    st = lib.kvs_check_evict_at(_ptr(evict_at), _ptr(cu_seqlens), B, T, ctypes.byref(fb), _stream(evict_at))
    if st == KVS_ERR_EVICT:
        return int(fb.value)
    _check("kvs_check_evict_at", st)
    return -1


def kvs_prof_enable(on: bool) -> None:
    lib.kvs_prof_enable(1 if on else 0)


def kvs_prof_reset() -> None:
    lib.kvs_prof_reset()


def kvs_prof_read(name: str) -> Tuple[int, float]:
    """(launches, total milliseconds) of the named kernel since the last reset."""
    n, ms = ctypes.c_int(0), ctypes.c_double(0.0)
    _check("kvs_prof_read", lib.kvs_prof_read(name.encode(), ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


class _EvictAttn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, evict_at, scale, cu_seqlens, max_seqlen):
        o, lse = kvs_evict_attn_fwd(q, k, v, evict_at, scale, cu_seqlens, max_seqlen)
        ctx.save_for_backward(q, k, v, o, lse, evict_at, cu_seqlens)
        ctx.scale, ctx.max_seqlen = scale, max_seqlen
        ctx.mark_non_differentiable(lse)
        ctx.set_materialize_grads(False)   # LSE carries no gradient: no zeros filled for it
        return o, lse

    @staticmethod
    def backward(ctx, do, _dlse):
        q, k, v, o, lse, evict_at, cu_seqlens = ctx.saved_tensors
        do = torch.zeros_like(o) if do is None else do
        dq, dk, dv = kvs_evict_attn_bwd(do.contiguous(), q, k, v, o, lse, evict_at, ctx.scale, cu_seqlens,
                                        ctx.max_seqlen)
        return dq, dk, dv, None, None, None, None


def evict_attn(q, k, v, evict_at, softmax_scale=None, cu_seqlens=None, max_seqlen=None):
    """Differentiable eviction-masked attention: returns ``(O, LSE)``; LSE carries no gradient."""
    scale = 1.0 / math.sqrt(q.shape[-1]) if softmax_scale is None else float(softmax_scale)
    return _EvictAttn.apply(q, k, v, evict_at, scale, cu_seqlens, max_seqlen)


# Gradients of a leaf are added up by one autograd node, which stays on the stream where the leaf was first used for as
# long as any graph of it lives.  If that is the default stream, a backward pass that is being captured would pull it
# into the capture, which ends the process; graphs of window_attn leave a mark on the node so that this can be refused.
_EAGER_MARK = "kvs: used on the default stream"


def _mark_eager(o: torch.Tensor) -> None:
    for node, _ in o.grad_fn.next_functions:
        if node is not None and not node.next_functions:   # a leaf's
            node.metadata[_EAGER_MARK] = True


def _refuse_captured(nodes) -> None:
    for node, _ in nodes:
        if node is not None and not node.next_functions and _EAGER_MARK in node.metadata:
            raise RuntimeError("window_attn: this backward is being captured, but an autograd graph made on the default "
                               "stream still uses the same leaves; let go of it before the capture")


class _WindowAttn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, sinks, evict_at, scale, cu_seqlens, max_seqlen, check_cu):
        rem = torch.empty_like(q, dtype=torch.int8) if any(ctx.needs_input_grad[:3]) else None
        o, lse = kvs_window_attn_fwd(q, k, v, window, sinks, evict_at, scale, cu_seqlens, max_seqlen, check_cu=check_cu,
                                     rem=rem)
        ctx.save_for_backward(q, k, v, o, rem, lse, evict_at, cu_seqlens)
        ctx.args = window, sinks, scale, max_seqlen
        ctx.mark_non_differentiable(lse)
        ctx.set_materialize_grads(False)   # LSE carries no gradient: no zeros filled for it
        return o, lse

    @staticmethod
    def backward(ctx, do, _dlse):
        # under create_graph a second derivative is refused, not zero (that wrapper takes 4 us)
        return (_window_grads_once if torch.is_grad_enabled() else _window_grads)(ctx, do)


def _window_grads(ctx, do):
    q, k, v, o, rem, lse, evict_at, cu_seqlens = ctx.saved_tensors
    window, sinks, scale, max_seqlen = ctx.args
    if torch.cuda.is_current_stream_capturing():
        _refuse_captured(ctx.next_functions)
    do = torch.zeros_like(o) if do is None else do
    # cu_seqlens is the forward's, which has checked it
    dq, dk, dv = kvs_window_attn_bwd(do.contiguous(), q, k, v, o, lse, window, sinks, evict_at, scale, cu_seqlens,
                                     max_seqlen, check_cu=False, rem=rem)
    return dq, dk, dv, None, None, None, None, None, None, None


_window_grads_once = torch.autograd.function.once_differentiable(_window_grads)


def window_attn(q, k, v, window: int, sinks: int = 0, evict_at=None, softmax_scale=None, cu_seqlens=None, max_seqlen=None,
                check_cu=True):
    """Differentiable attention under a sliding window with sinks: returns ``(O, LSE)``; LSE carries no gradient."""
    scale = 1.0 / math.sqrt(q.shape[-1]) if softmax_scale is None else float(softmax_scale)
    o, lse = _WindowAttn.apply(q, k, v, int(window), int(sinks), evict_at, scale, cu_seqlens, max_seqlen, check_cu)
    if o.requires_grad and _stream(q) == 0:
        _mark_eager(o)
    return o, lse
