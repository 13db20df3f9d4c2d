"""Operators around the linear layers (argument marshalling only): the root-mean-square norm
with the residual's addition, in values or as quantized operands, its gradient, and the 2-norm of
gradients with clipping.  The definitions stand in ``include/q2d.h``."""
from __future__ import annotations

import array
import ctypes
import operator
import struct

import torch

from . import FP4_1D, FP4_2D, MXFP8, Q2DError, QTensor, _check, _DTYPE_CODES, _dtype_code, _lib, _same_device, _stream, _Tensor


class _Norm(ctypes.Structure):
    _fields_ = [("x_dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32),
                ("y_dtype", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("eps", ctypes.c_double),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("residual", ctypes.c_void_p),
                ("ld_residual", ctypes.c_int64), ("weight", ctypes.c_void_p), ("h", ctypes.c_void_p),
                ("ldh", ctypes.c_int64), ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64), ("rstd", ctypes.c_void_p)]


class _NormGrad(ctypes.Structure):
    _fields_ = [("h_dtype", ctypes.c_int32), ("dy_dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("h", ctypes.c_void_p), ("ldh", ctypes.c_int64), ("dy", ctypes.c_void_p), ("lddy", ctypes.c_int64),
                ("dh", ctypes.c_void_p), ("lddh", ctypes.c_int64), ("dx", ctypes.c_void_p), ("lddx", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("rstd", ctypes.c_void_p), ("dw", ctypes.c_void_p)]


# the same structures, packed
_NORM = struct.Struct("4i2qdQqQqQQqQqQ")
_GRAD = struct.Struct("3i4x2qQqQqQqQqQQQ")
assert _NORM.size == ctypes.sizeof(_Norm) and _GRAD.size == ctypes.sizeof(_NormGrad)

_P, _I64, _I32, _F64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double
_TP = ctypes.POINTER(_Tensor)
for _name, _args, _res in (
        ("q2d_rmsnorm_fwd", [_P, _TP, _TP, _P], _I32),
        ("q2d_rmsnorm_workspace", [_I64, _I64], _I64),
        ("q2d_rmsnorm_bwd", [_P, _P, _I64, _P], _I32),
        ("q2d_grad_workspace", [_I32], _I64),
        ("q2d_grad_norm", [_I32, _P, _P, _P, _P, _P, _I64, _P], _I32),
        ("q2d_clip_grads", [_I32, _P, _P, _P, _P, _F64, _P, _P, _P, _I64, _P], _I32)):
    getattr(_lib, _name).argtypes, getattr(_lib, _name).restype = _args, _res


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _call(device, name, *args):
    """A call of the library on the device's current stream, with the device made current."""
    if device.index is not None and device.index != _current_device():
        with torch.cuda.device(device):
            return _check(getattr(_lib, name)(*args, _stream(device)), name)
    _check(getattr(_lib, name)(*args, _stream(device)), name)


def _modified(tensors):
    """Tells autograd of the caller's tensors (None: none) that a call has written: a backward pass
    that needs their old values is refused."""
    written = [t for t in tensors if t is not None]
    if written:
        torch.autograd.graph.increment_version(written)


def _rows(t, shape, device, what):
    """(pointer, row pitch) of a [rows, cols] tensor with unit stride along its rows."""
    if t.shape != shape:
        raise Q2DError("%s: a tensor of shape %s is expected" % (what, tuple(shape)))
    pitch, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise Q2DError("%s: unit stride along the rows is expected" % what)
    if t.device != device:
        _same_device(device, t)
    return t.data_ptr(), pitch


def _vector(t, n, device, what, dtype=None):
    if t.shape != (n,) or not t.is_contiguous() or (dtype is not None and t.dtype != dtype):
        raise Q2DError("%s: a contiguous %s vector of %d elements is expected" % (what, dtype or "device", n))
    if t.device != device:
        _same_device(device, t)
    return t.data_ptr()


def _forward(x, weight, eps, residual, h, rstd, y, q4, q8):
    """q2d_rmsnorm_fwd, with h and rstd made where they are None; returns them."""
    device, shape = x.device, x.shape
    if device.type != "cuda" or len(shape) != 2:
        raise Q2DError("expected x as a 2-D device tensor")
    rows, cols = shape
    xp, ldx = _rows(x, shape, device, "x")
    rp = ldr = hp = ldh = yp = ldy = r_code = y_code = 0
    x_code = _dtype_code(x.dtype)
    if residual is not None:
        if h is None:
            h = torch.empty_like(x, memory_format=torch.contiguous_format)
        elif h.dtype != x.dtype:
            raise Q2DError("h: the dtype of x is expected")
        r_code = _dtype_code(residual.dtype)
        rp, ldr = _rows(residual, shape, device, "residual")
        hp, ldh = _rows(h, shape, device, "h")
    elif h is not None:
        raise Q2DError("h is x itself without a residual")
    else:
        h = x
    if y is not None:
        y_code = _dtype_code(y.dtype)
        yp, ldy = _rows(y, shape, device, "y")
    if rstd is None:
        rstd = torch.empty(rows, dtype=torch.float32, device=device)
        sp = rstd.data_ptr()
    else:
        sp = _vector(rstd, rows, device, "rstd", torch.float32)
    # (packed: a ctypes structure filled field by field takes 2 us more)
    _call(device, "q2d_rmsnorm_fwd",
          _NORM.pack(x_code, r_code, _dtype_code(weight.dtype), y_code, rows, cols, eps, xp, ldx, rp, ldr,
                     _vector(weight, cols, device, "weight"), hp, ldh, yp, ldy, sp), q4, q8)
    return h, rstd


def q2d_rmsnorm_fwd(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5, residual: torch.Tensor | None = None,
                    y_dtype=torch.bfloat16, y: torch.Tensor | None = None, h: torch.Tensor | None = None,
                    rstd: torch.Tensor | None = None):
    """Root-mean-square norm of the rows of h = x + residual (x [rows, cols]; h in x's dtype, x
    itself without a residual) times weight [cols]; returns (y, h, rstd).  rstd (float32 [rows])
    is what q2d_rmsnorm_bwd needs.  h may be x or residual itself: in place.  Tensors handed in as
    y, h and rstd count as modified for autograd."""
    given = y, h, rstd
    if y is None:
        y = torch.empty_like(x, dtype=y_dtype, memory_format=torch.contiguous_format)
    h, rstd = _forward(x, weight, eps, residual, h, rstd, y, None, None)
    _modified(given)
    return y, h, rstd


def q2d_rmsnorm_quantize(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5, residual: torch.Tensor | None = None,
                         formats=(FP4_2D,), block: int = 32, orientations=(True, True), out=None,
                         h: torch.Tensor | None = None, rstd: torch.Tensor | None = None):
    """q2d_rmsnorm_fwd with y as operands of the linear layers' GEMMs in place of values: one
    QTensor for each of ``formats`` (one of FP4_2D and FP4_1D, MXFP8, or both), from one read of
    h; returns (list of QTensors, h, rstd).  The codes are those of the quantizers for the
    float32 y, rounded to nearest.  block: edge of the 2D blocks (32 or 64); orientations: (True,
    False) for the rowwise copies alone, which a forward GEMM reads; out: QTensors to fill.  h and
    rstd handed in count as modified for autograd."""
    formats = tuple(formats)
    kinds = [f == MXFP8 for f in formats]
    if not formats or any(f not in (FP4_2D, FP4_1D, MXFP8) for f in formats) or len(set(kinds)) != len(kinds):
        raise Q2DError("formats: one of FP4_2D and FP4_1D, MXFP8, or one of each is expected")
    if x.dim() != 2:
        raise Q2DError("expected x as a 2-D device tensor")
    if out is None:
        out = [QTensor(f, *x.shape, x.device, block if f == FP4_2D else 32, orientations) for f in formats]
    else:
        if len(out) != len(formats) or any(q.fmt != f or q.nseg is not None for q, f in zip(out, formats)):
            raise Q2DError("out: a QTensor for each of formats is expected")
        _same_device(x.device, *out)
    q = [None, None]
    for t, mx in zip(out, kinds):
        q[mx] = t.ptr()
    given = h, rstd
    h, rstd = _forward(x, weight, eps, residual, h, rstd, None, *q)
    _modified(given)
    return out, h, rstd


def q2d_rmsnorm_bwd(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor,
                    dh: torch.Tensor | None = None, dx: torch.Tensor | None = None, dw: torch.Tensor | None = None,
                    need_dw: bool = True):
    """Gradients (dx, dw) of the norm from dy, and h and rstd of the forward call: dx (h's dtype)
    for x and for the residual, with dh, the gradient that reaches h by other ways, added; dw
    (float32 [cols]) for the weight, None with need_dw=False.  dx may be dh itself.  dx and dw handed
    in count as modified for autograd."""
    given = dx, dw
    device, shape = h.device, h.shape
    if device.type != "cuda" or len(shape) != 2:
        raise Q2DError("expected h as a 2-D device tensor")
    rows, cols = shape
    if dx is None:
        dx = torch.empty_like(h, memory_format=torch.contiguous_format)
    if dx.dtype != h.dtype or (dh is not None and dh.dtype != h.dtype):
        raise Q2DError("dh and dx: the dtype of h is expected")
    dhp = lddh = wp = 0
    if dh is not None:
        dhp, lddh = _rows(dh, shape, device, "dh")
    if need_dw:
        if dw is None:
            dw = torch.empty(cols, dtype=torch.float32, device=device)
        wp = _vector(dw, cols, device, "dw", torch.float32)
    elif dw is not None:
        raise Q2DError("dw is not computed with need_dw=False")
    size = max(_lib.q2d_rmsnorm_workspace(rows, cols), 0)
    ws = torch.empty(size, dtype=torch.uint8, device=device)
    _call(device, "q2d_rmsnorm_bwd",
          _GRAD.pack(_dtype_code(h.dtype), _dtype_code(dy.dtype), _dtype_code(weight.dtype), rows, cols,
                     *_rows(h, shape, device, "h"), *_rows(dy, shape, device, "dy"), dhp, lddh,
                     *_rows(dx, shape, device, "dx"), _vector(weight, cols, device, "weight"),
                     _vector(rstd, rows, device, "rstd", torch.float32), wp), ws.data_ptr(), size)
    _modified(given)
    return dx, dw


_DTYPE_OF = operator.attrgetter("dtype")


def _dense(t):
    """Whether t's elements lie without gaps or overlaps, in any order of the dimensions."""
    span = 1
    for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n > 1):
        if stride != span:
            return False
        span *= size
    return True


def _gradients(tensors, what):
    """A list of tensors, their pointers, counts and dtypes as arrays for the C ABI, and whether all
    are contiguous."""
    tensors = list(tensors)
    if not tensors:
        raise Q2DError("%s: a list of device tensors is expected" % what)
    try:
        dense = all(map(torch.Tensor.is_contiguous, tensors))
    except TypeError:
        raise Q2DError("%s: a list of device tensors is expected" % what) from None
    if not dense and not all(map(_dense, tensors)):
        raise Q2DError("%s: tensors without gaps are expected" % what)
    devices = set(map(torch.Tensor.get_device, tensors))
    if len(devices) > 1 or min(devices) < 0:
        raise Q2DError("%s: tensors on one device are expected" % what)
    kinds = set(map(_DTYPE_OF, tensors))
    if not kinds <= _DTYPE_CODES.keys():
        raise Q2DError("%s: float32 or bfloat16 tensors are expected" % what)
    if len(kinds) == 1:
        dtypes = array.array("i", [_DTYPE_CODES[kinds.pop()]]) * len(tensors)
    else:
        dtypes = array.array("i", [_DTYPE_CODES[t.dtype] for t in tensors])
    # (from lists: an array grown element by element takes a quarter longer)
    pointers = array.array("Q", list(map(torch.Tensor.data_ptr, tensors)))
    counts = array.array("q", list(map(torch.Tensor.numel, tensors)))
    return tensors, pointers, counts, dtypes, dense


def _address(a):
    return a.buffer_info()[0]


def q2d_grad_norm(tensors, norm: torch.Tensor | None = None) -> torch.Tensor:
    """2-norm over all elements of a list of tensors (float32 or bfloat16, without gaps), as a
    float32 device scalar.  A norm handed in counts as modified for autograd."""
    tensors, pointers, counts, dtypes, _ = _gradients(tensors, "tensors")
    device, given = tensors[0].device, norm
    norm = _scalar(norm, device, "norm")
    size = _lib.q2d_grad_workspace(len(tensors))
    ws = torch.empty(size, dtype=torch.uint8, device=device)
    _call(device, "q2d_grad_norm", len(tensors), _address(pointers), _address(counts), _address(dtypes), norm.data_ptr(),
          ws.data_ptr(), size)
    _modified((given,))
    return norm


def _scalar(t, device, what):
    if t is None:
        return torch.empty((), dtype=torch.float32, device=device)
    if t.dtype != torch.float32 or t.numel() != 1:
        raise Q2DError("%s: a float32 scalar is expected" % what)
    _same_device(device, t)
    return t


def q2d_clip_grads(tensors, max_norm: float, norm: torch.Tensor | None = None, out=None) -> torch.Tensor:
    """Scales a list of tensors by min(1, max_norm / norm), in place or into the tensors of
    ``out``; returns the norm (float32 device scalar).  norm: the value to go by, the 2-norm over
    tensors of several GPUs for one; None: that of q2d_grad_norm.  A norm that is not finite
    leaves the values as they are.  Nothing waits for the device.  The tensors that are written count
    as modified for autograd, whatever the norm is."""
    tensors, pointers, counts, dtypes, dense = _gradients(tensors, "tensors")
    device = tensors[0].device
    outs = None
    if out is not None:
        out, outs, out_counts, out_dtypes, out_dense = _gradients(out, "out")
        # (contiguous ones need the same number of elements only)
        if out_dtypes != dtypes or out_counts != counts or out[0].device != device or (
                not (dense and out_dense) and any(a.shape != b.shape or a.stride() != b.stride() for a, b in zip(out, tensors))):
            raise Q2DError("out: a tensor like each of tensors is expected")
    given = norm
    norm = _scalar(norm, device, "norm")
    size = 0 if given is not None else _lib.q2d_grad_workspace(len(tensors))
    ws = torch.empty(size, dtype=torch.uint8, device=device)
    _call(device, "q2d_clip_grads", len(tensors), _address(pointers), None if outs is None else _address(outs),
          _address(counts), _address(dtypes), float(max_norm), None if given is None else norm.data_ptr(),
          norm.data_ptr() if given is None else None, ws.data_ptr(), size)
    # (behind the launches, while the device is at work: 6 us of 240 tensors)
    torch.autograd.graph.increment_version(tensors if out is None else out)
    return norm
