"""Attention operators of the binding (argument marshalling only): whole sequences forward
and backward.  The definitions stand in ``include/q2d.h``."""
from __future__ import annotations

import ctypes
import functools
import math

import torch

from . import Q2DError, _check, _dtype_code, _lib, _same_device, _stream


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_batch", ctypes.c_int64),
                ("stride_length", ctypes.c_int64), ("stride_head", ctypes.c_int64)]


class _Attention(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("len_q", ctypes.c_int64), ("len_k", ctypes.c_int64), ("window", ctypes.c_int64),
                ("scale", ctypes.c_float), ("softcap", ctypes.c_float),
                ("slopes", ctypes.c_void_p), ("documents", ctypes.c_void_p), ("prefix", ctypes.c_void_p),
                ("q", _Heads), ("k", _Heads), ("v", _Heads), ("out", _Heads), ("lse", ctypes.c_void_p)]


_P, _I64, _I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
_AP, _HP = ctypes.POINTER(_Attention), ctypes.POINTER(_Heads)
_lib.q2d_attention_workspace.argtypes, _lib.q2d_attention_workspace.restype = [_AP, _I32], _I64
_lib.q2d_attention_fwd.argtypes, _lib.q2d_attention_fwd.restype = [_AP, _P, _I64, _P], _I32
_lib.q2d_attention_bwd.argtypes, _lib.q2d_attention_bwd.restype = [_AP, _HP, _HP, _HP, _HP, _P, _I64, _P], _I32


def _vector(t, n, dtype, device, what):
    """Pointer of an optional contiguous device vector or matrix of n elements."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise Q2DError("%s: a contiguous %s tensor of %d elements is expected" % (what, dtype, n))
    _same_device(device, t)
    return t.data_ptr()


def _heads(t, shape, dtype, device, what, into=None):
    """Descriptor of a [batch, length, heads, dim] tensor (any strides, unit along dim)."""
    if tuple(t.shape) != shape or t.dtype != dtype or (t.stride(3) != 1 and shape[3] > 1):
        raise Q2DError("%s: a %s tensor of shape %s with unit stride along the last dimension is expected"
                       % (what, dtype, shape))
    _same_device(device, t)
    d = _Heads() if into is None else into
    d.data = t.data_ptr()
    d.stride_batch, d.stride_length, d.stride_head = t.stride(0), t.stride(1), t.stride(2)
    return d


@functools.lru_cache(maxsize=1024)
def _template(dtype, causal, batch, heads_q, heads_kv, dim, len_q, len_k, window, scale, softcap, documents):
    """Descriptor of a problem without its pointers, and both workspace sizes."""
    a = _Attention(dtype=dtype, causal=causal, batch=batch, heads_q=heads_q, heads_kv=heads_kv, dim=dim, len_q=len_q,
                   len_k=len_k, window=window, scale=scale, softcap=softcap)
    a.documents = 256 if documents else None
    sizes = [_lib.q2d_attention_workspace(ctypes.byref(a), i) for i in (0, 1)]
    a.documents = None
    return bytes(a), sizes


def _problem(q, k, v, out, lse, scale, causal, window, softcap, slopes, documents, prefix):
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise Q2DError("expected q, k and v as [batch, length, heads, dim]")
    B, Lq, Hq, D = q.shape
    Lk, Hkv = k.shape[1], k.shape[2]
    device, dt = q.device, q.dtype
    _same_device(device)
    if scale is None:
        scale = 1.0 / math.sqrt(D) if D else 0.0
    raw, sizes = _template(_dtype_code(dt), int(bool(causal)), B, Hq, Hkv, D, Lq, Lk, int(window), float(scale),
                           float(softcap), documents is not None)
    a = _Attention.from_buffer_copy(raw)
    kv = (B, Lk, Hkv, D)
    _heads(q, (B, Lq, Hq, D), dt, device, "q", a.q)
    _heads(k, kv, dt, device, "k", a.k)
    _heads(v, kv, dt, device, "v", a.v)
    _heads(out, (B, Lq, Hq, D), dt, device, "out", a.out)
    a.slopes = _vector(slopes, Hq, torch.float32, device, "slopes")
    a.documents = _vector(documents, B * Lk, torch.int32, device, "documents")
    a.prefix = _vector(prefix, B, torch.int32, device, "prefix")
    a.lse = _vector(lse, B * Hq * Lq, torch.float32, device, "lse")
    return a, sizes


def _workspace(size, device):
    """(tensor, pointer) of a call's workspace; None for none or for invalid sizes, which
    the call itself reports."""
    if size <= 0:
        return None, None
    t = torch.empty(size, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def q2d_attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float | None = None, causal: bool = True,
                      window: int = 0, softcap: float = 0.0, slopes: torch.Tensor | None = None,
                      documents: torch.Tensor | None = None, prefix: torch.Tensor | None = None,
                      out: torch.Tensor | None = None, need_lse: bool = True):
    """Attention of q [batch, len_q, heads_q, dim] on k, v [batch, len_k, heads_kv, dim];
    returns (out, lse).  Queries are the last len_q positions of the sequence.

    scale defaults to dim ** -0.5.  softcap > 0 caps scores by softcap * tanh(s / softcap);
    slopes (float32 [heads_q]) subtracts slope * distance; window > 0 leaves distances below
    it; documents (int32 [batch, len_k], negative: padding) keeps attention within documents;
    prefix (int32 [batch]) lets every query see the first keys.  lse (float32 [batch,
    heads_q, len_q]) is what q2d_attention_bwd needs, None with need_lse=False."""
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = None
    if need_lse and q.dim() == 4:
        lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
    a, sizes = _problem(q, k, v, out, lse, scale, causal, window, softcap, slopes, documents, prefix)
    keep, ws = _workspace(sizes[0], q.device)
    _check(_lib.q2d_attention_fwd(ctypes.byref(a), ws, max(sizes[0], 0), _stream(q.device)), "q2d_attention_fwd")
    return out, lse


def q2d_attention_bwd(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                      lse: torch.Tensor, scale: float | None = None, causal: bool = True, window: int = 0,
                      softcap: float = 0.0, slopes: torch.Tensor | None = None, documents: torch.Tensor | None = None,
                      prefix: torch.Tensor | None = None, dq: torch.Tensor | None = None,
                      dk: torch.Tensor | None = None, dv: torch.Tensor | None = None):
    """Gradients (dq, dk, dv) of q2d_attention_fwd with the same arguments, from its out and
    lse and the gradient dout of out."""
    a, sizes = _problem(q, k, v, out, lse, scale, causal, window, softcap, slopes, documents, prefix)
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=q.dtype, device=q.device) if dk is None else dk
    dv = torch.empty(k.shape, dtype=q.dtype, device=q.device) if dv is None else dv
    g = [_heads(t, tuple(s.shape), q.dtype, q.device, n)
         for t, s, n in ((dout, q, "dout"), (dq, q, "dq"), (dk, k, "dk"), (dv, k, "dv"))]
    keep, ws = _workspace(sizes[1], q.device)
    _check(_lib.q2d_attention_bwd(ctypes.byref(a), *[ctypes.byref(x) for x in g], ws, max(sizes[1], 0),
                                  _stream(q.device)), "q2d_attention_bwd")
    return dq, dk, dv
