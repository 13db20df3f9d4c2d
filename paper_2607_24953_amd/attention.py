"""Attention operators of the binding (argument marshalling only): whole sequences forward
and backward, and new tokens over a paged 8-bit key/value cache.  The definitions stand in
``include/q2d.h``."""
from __future__ import annotations

import ctypes
import functools

import torch

from . import Q2DError, _check, _dtype_code, _lib, _norm, _same_device, _stream


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


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int32), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("k_codes", ctypes.c_void_p), ("v_codes_t", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


class _Sequences(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("table_pages", ctypes.c_int32), ("tokens", ctypes.c_int64),
                ("table_stride", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("table", ctypes.c_void_p)]


class _CachedAttention(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("scale", ctypes.c_float),
                ("softcap", ctypes.c_float), ("window", ctypes.c_int64), ("slopes", ctypes.c_void_p),
                ("prefix", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("q_stride_token", ctypes.c_int64), ("q_stride_head", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("out_stride_token", ctypes.c_int64), ("out_stride_head", ctypes.c_int64)]


_P, _I64, _I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
_AP = ctypes.POINTER(_Attention)
_lib.q2d_attention_workspace.argtypes, _lib.q2d_attention_workspace.restype = [_AP, _I32], _I64
_lib.q2d_attention_fwd.argtypes, _lib.q2d_attention_fwd.restype = [_AP, _P, _I64, _P], _I32
# (the four descriptors stand in one array)
_lib.q2d_attention_bwd.argtypes, _lib.q2d_attention_bwd.restype = [_AP, _P, _P, _P, _P, _P, _I64, _P], _I32

_CP, _SP = ctypes.POINTER(_Cache), ctypes.POINTER(_Sequences)
_lib.q2d_kv_cache_init.argtypes = [_CP, _I32, _I32, _I32, _I32, ctypes.POINTER(_I64)]
_lib.q2d_kv_cache_init.restype = _I32
for _name in ("q2d_kv_write", "q2d_kv_read"):
    getattr(_lib, _name).argtypes = [_CP, _SP, _I32, _P, _I64, _I64, _P, _I64, _I64, _P]
    getattr(_lib, _name).restype = _I32
_lib.q2d_attention_cached_workspace.argtypes, _lib.q2d_attention_cached_workspace.restype = [_CP, _SP, _I32], _I64
_lib.q2d_attention_cached.argtypes = [_CP, _SP, ctypes.POINTER(_CachedAttention), _P, _I64, _P]
_lib.q2d_attention_cached.restype = _I32


def _on(device, t):
    if t.device != device:
        _same_device(device, t)


def _vector(t, n, dtype, device, what, shape=None):
    """Pointer of an optional contiguous device vector of n elements, or a tensor of ``shape``."""
    if t is None:
        return None
    if shape is not None and t.dim() != 1 and t.shape != shape:
        raise Q2DError("%s: a tensor of shape %s is expected" % (what, shape))
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise Q2DError("%s: a contiguous %s tensor of %d elements is expected" % (what, dtype, n))
    _on(device, t)
    return t.data_ptr()


def _heads(t, shape, dtype, device, what, d):
    """Fills descriptor d of a [batch, length, heads, dim] tensor (any strides, unit along dim)."""
    st = t.stride()
    if t.shape != shape or t.dtype != dtype or (st[3] != 1 and shape[3] > 1):
        raise Q2DError("%s: a %s tensor of shape %s with unit stride along the last dimension is expected"
                       % (what, dtype, tuple(shape)))
    _on(device, t)
    d.data = t.data_ptr()
    d.stride_batch, d.stride_length, d.stride_head = st[0], st[1], st[2]


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
    if q.dim() != 4 or k.dim() != 4:
        raise Q2DError("expected q, k and v as [batch, length, heads, dim]")
    qs, ks = q.shape, k.shape
    B, Lq, Hq, D = qs
    Lk, Hkv = ks[1], ks[2]
    device, dt = q.device, q.dtype
    if device.type != "cuda" or ks[0] != B or ks[3] != D:
        _same_device(device)
        raise Q2DError("k: a tensor of shape %s is expected" % ((B, Lk, Hkv, D),))
    if scale is None:
        scale = D ** -0.5 if D else 0.0
    raw, sizes = _template(_dtype_code(dt), 1 if causal else 0, B, Hq, Hkv, D, Lq, Lk, int(window), float(scale),
                           float(softcap), documents is not None)
    a = _Attention.from_buffer_copy(raw)
    _heads(q, qs, dt, device, "q", a.q)
    _heads(k, ks, dt, device, "k", a.k)
    _heads(v, ks, dt, device, "v", a.v)
    _heads(out, qs, dt, device, "out", a.out)
    if slopes is not None:
        a.slopes = _vector(slopes, Hq, torch.float32, device, "slopes")
    if documents is not None:
        a.documents = _vector(documents, B * Lk, torch.int32, device, "documents", (B, Lk))
    if prefix is not None:
        a.prefix = _vector(prefix, B, torch.int32, device, "prefix")
    a.lse = _vector(lse, B * Hq * Lq, torch.float32, device, "lse", (B, Hq, Lq))
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
    if q.dim() != 4 or v.dim() != 4 or (out is not None and out.dim() != 4):
        raise Q2DError("expected q, k and v as [batch, length, heads, dim]")
    shape = q.shape
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=q.device)
    lse = None
    if need_lse:
        lse = torch.empty((shape[0], shape[2], shape[1]), dtype=torch.float32, device=q.device)
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
    if v.dim() != 4 or out.dim() != 4:
        raise Q2DError("expected v and out as [batch, length, heads, dim]")
    a, sizes = _problem(q, k, v, out, lse, scale, causal, window, softcap, slopes, documents, prefix)
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=q.dtype, device=q.device) if dk is None else dk
    dv = torch.empty(k.shape, dtype=q.dtype, device=q.device) if dv is None else dv
    g = (_Heads * 4)()
    for i, (t, s, n) in enumerate(((dout, q, "dout"), (dq, q, "dq"), (dk, k, "dk"), (dv, k, "dv"))):
        if t.dim() != 4:
            raise Q2DError("%s: a [batch, length, heads, dim] tensor is expected" % n)
        _heads(t, s.shape, q.dtype, q.device, n, g[i])
    size = ctypes.sizeof(_Heads)
    keep, ws = _workspace(sizes[1], q.device)
    _check(_lib.q2d_attention_bwd(ctypes.byref(a), ctypes.byref(g), ctypes.byref(g, size), ctypes.byref(g, 2 * size),
                                  ctypes.byref(g, 3 * size), ws, max(sizes[1], 0), _stream(q.device)),
           "q2d_attention_bwd")
    return dq, dk, dv


class KVCache:
    """A paged key/value cache in 8 bits: E4M3 codes with one power-of-two scale for each
    block of 32 tokens and head.  ``pages`` pages of ``page_size`` tokens (a multiple of 32)
    are shared by all sequences; which page holds which tokens is the caller's page table.

    ``k_codes`` [pages, heads, page_size, dim], ``v_codes_t`` [pages, heads, page_size / 32,
    dim, 32] (values transposed in their block), ``k_scales`` and ``v_scales`` [pages, heads,
    page_size / 32], all uint8 and zeroed here."""

    def __init__(self, pages: int, heads: int, dim: int, page_size: int = 64, device="cuda"):
        self.desc = _Cache()
        _check(_lib.q2d_kv_cache_init(ctypes.byref(self.desc), int(pages), int(heads), int(dim), int(page_size), None),
               "q2d_kv_cache_init")
        self._ref = ctypes.byref(self.desc)
        self.pages, self.heads, self.dim, self.page_size = int(pages), int(heads), int(dim), int(page_size)
        self.device = _norm(device)
        self.scale = self.dim ** -0.5
        blocks = self.page_size // 32
        shapes = {"k_codes": (pages, heads, page_size, dim), "v_codes_t": (pages, heads, blocks, dim, 32),
                  "k_scales": (pages, heads, blocks), "v_scales": (pages, heads, blocks)}
        for name, shape in shapes.items():
            t = torch.zeros(shape, dtype=torch.uint8, device=self.device)
            setattr(self, name, t)
            setattr(self.desc, name, t.data_ptr())


@functools.lru_cache(maxsize=1024)
def _sequences_template(batch, table_pages, tokens, table_stride):
    return bytes(_Sequences(batch=batch, table_pages=table_pages, tokens=tokens, table_stride=table_stride))


def _sequences(cache, table, lens, tokens, offsets):
    if not isinstance(cache, KVCache):
        raise Q2DError("expected a KVCache")
    if cache.device.type != "cuda":
        _same_device(cache.device)
    if table.dim() != 2 or table.dtype != torch.int32:
        raise Q2DError("block_table: an int32 tensor [sequences, pages] is expected")
    batch, pages = table.shape
    stride, one = table.stride()
    if one != 1 and pages > 1:
        raise Q2DError("block_table: unit column stride is expected")
    _on(cache.device, table)
    s = _Sequences.from_buffer_copy(_sequences_template(batch, pages, tokens, stride if batch > 1 else max(stride, pages)))
    s.table = table.data_ptr()
    s.lens = _vector(lens, batch, torch.int32, cache.device, "lens")
    if offsets is not None:
        s.offsets = _vector(offsets, batch + 1, torch.int64, cache.device, "offsets")
    return s


def _token_rows(t, heads, dim, device, what):
    shape, st = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim or st[2] != 1:
        raise Q2DError("%s: a [tokens, %d, %d] tensor with unit stride along the last dimension is expected"
                       % (what, heads, dim))
    _on(device, t)
    return t.data_ptr(), st[0], st[1]


@functools.lru_cache(maxsize=1024)
def _cached_template(dtype, heads, scale, softcap, window):
    return bytes(_CachedAttention(dtype=dtype, heads_q=heads, scale=scale, softcap=softcap, window=window))


@functools.lru_cache(maxsize=1024)
def _cached_workspace(pages, heads, dim, page_size, sequences, offsets, heads_q):
    c, s = _Cache(pages=pages, heads=heads, dim=dim, page_size=page_size), _Sequences.from_buffer_copy(sequences)
    s.offsets = 256 if offsets else None
    return _lib.q2d_attention_cached_workspace(ctypes.byref(c), ctypes.byref(s), heads_q)


def q2d_kv_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor,
                 offsets: torch.Tensor | None = None) -> KVCache:
    """Append the tokens of k and v [tokens, heads, dim] to the cache.

    lens (int32 [sequences]) counts each sequence's tokens with the new ones; the new ones are
    rows offsets[b] .. offsets[b + 1] (int64 [sequences + 1]; None: equally many each, in
    order).  block_table (int32 [sequences, pages]) names the pages."""
    if k.dim() != 3 or k.shape != v.shape or k.dtype != v.dtype:
        raise Q2DError("expected k and v as [tokens, heads, dim] of one dtype")
    s = _sequences(cache, block_table, lens, k.shape[0], offsets)
    _check(_lib.q2d_kv_write(cache._ref, ctypes.byref(s), _dtype_code(k.dtype),
                             *_token_rows(k, cache.heads, cache.dim, cache.device, "k"),
                             *_token_rows(v, cache.heads, cache.dim, cache.device, "v"), _stream(cache.device)),
           "q2d_kv_write")
    return cache


def q2d_kv_read(cache: KVCache, block_table: torch.Tensor, lens: torch.Tensor, tokens: int,
                offsets: torch.Tensor | None = None, out_dtype=torch.float32,
                k: torch.Tensor | None = None, v: torch.Tensor | None = None):
    """Values (k, v) [tokens, heads, dim] of each sequence's last tokens (offsets as in
    q2d_kv_write, ``tokens`` in all); zeros in rows of no sequence, before a sequence's first
    token and on pages that the table does not name."""
    shape = (int(tokens), cache.heads, cache.dim)
    k = torch.empty(shape, dtype=out_dtype, device=cache.device) if k is None else k
    v = torch.empty(shape, dtype=k.dtype, device=cache.device) if v is None else v
    if k.shape != v.shape or k.dtype != v.dtype or k.dim() != 3 or k.shape[0] != int(tokens):
        raise Q2DError("expected k and v as [tokens, heads, dim] of one dtype")
    s = _sequences(cache, block_table, lens, int(tokens), offsets)
    _check(_lib.q2d_kv_read(cache._ref, ctypes.byref(s), _dtype_code(k.dtype),
                            *_token_rows(k, cache.heads, cache.dim, cache.device, "k"),
                            *_token_rows(v, cache.heads, cache.dim, cache.device, "v"), _stream(cache.device)),
           "q2d_kv_read")
    return k, v


def q2d_attention_cached(q: torch.Tensor, cache: KVCache, block_table: torch.Tensor, lens: torch.Tensor,
                         offsets: torch.Tensor | None = None, scale: float | None = None, window: int = 0,
                         softcap: float = 0.0, slopes: torch.Tensor | None = None,
                         prefix: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Causal attention of each sequence's last tokens, q [tokens, heads_q, dim] in bfloat16,
    over its keys and values in the cache, these tokens' own among them.  offsets, lens and
    block_table as in q2d_kv_write; scale, window, softcap, slopes and prefix as in
    q2d_attention_fwd.  Rows outside offsets[0] .. offsets[-1] (a padded batch) are zeros."""
    if q.dim() != 3:
        raise Q2DError("expected q as [tokens, heads, dim]")
    tokens, heads, _ = q.shape
    s = _sequences(cache, block_table, lens, tokens, offsets)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif out.dtype != q.dtype or out.shape != q.shape:
        raise Q2DError("out: the shape and dtype of q are expected")
    device = cache.device
    a = _CachedAttention.from_buffer_copy(_cached_template(
        _dtype_code(q.dtype), heads, cache.scale if scale is None else float(scale), float(softcap), int(window)))
    if slopes is not None:
        a.slopes = _vector(slopes, heads, torch.float32, device, "slopes")
    if prefix is not None:
        a.prefix = _vector(prefix, s.batch, torch.int32, device, "prefix")
    a.q, a.q_stride_token, a.q_stride_head = _token_rows(q, heads, cache.dim, device, "q")
    a.out, a.out_stride_token, a.out_stride_head = _token_rows(out, heads, cache.dim, device, "out")
    size = _cached_workspace(cache.pages, cache.heads, cache.dim, cache.page_size,
                             _sequences_template(s.batch, s.table_pages, tokens, s.table_stride), offsets is not None, heads)
    keep, ws = _workspace(size, device)
    _check(_lib.q2d_attention_cached(cache._ref, ctypes.byref(s), ctypes.byref(a), ws, max(size, 0), _stream(device)),
           "q2d_attention_cached")
    return out
