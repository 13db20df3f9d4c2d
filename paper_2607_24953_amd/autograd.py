"""PyTorch autograd forms: the quantized linear layer (Sec. 3; App. C, App. E), alone or behind a
root-mean-square norm, that norm by itself, and attention.

``Q2DLinear`` is a bias-free linear layer y = x W^T whose forward and backward
GEMMs run on quantized operands through ``q2d_linear_fwd`` / ``q2d_linear_bwd``:

* forward: X and W are quantized (round to nearest by default, the forward
  placement of App. E), Y = Q(X) Q(W)^T;
* backward: dY is quantized (stochastic rounding by default, App. E) and
  dX = Q(dY) Q(W), dW = Q(dY)^T Q(X) reuse the forward's quantized copies
  transposed (the 2D blocks keep their scales; Sec. 3);
* the straight-through estimator (Sec. 3) treats the quantizer as the identity:
  the gradients above are returned for x and W as they are.

Each call draws fresh stochastic-rounding streams: the layer's seed with
offsets 3n, 3n+1, 3n+2 for X, W and dY of its n-th forward call.  A layer built
without a seed takes the next value of a process-wide counter, so the layers of
a model draw independent streams (App. E asks for unbiased, independent
rounding; one seed shared by every layer would give the n-th gradients of all
layers the same random bits at the same storage indices).  The weight
(the master copy, usually float32) is cast to the input's dtype (float32 or
bfloat16) before quantization; Y and dX have the input's dtype, dW is computed
in float32 and cast to the weight's dtype.

``Q2DNormLinear`` is the same layer on norm(x + residual): q2d_rmsnorm_quantize writes the
GEMMs' operand, so X is neither written nor read in 16 bits, and Q(X) is rounded once, from
float32.  ``rms_norm`` gives the normed values themselves.  Both return the sum x + residual
beside their output, for the residual stream, and their backward takes its gradient in the
same pass (q2d_rmsnorm_bwd).

A backward pass can be captured into a HIP graph.  Let go of every eager output of the same
parameters first: torch keeps their gradients' accumulation on the eager stream for as long as one
lives, and a capture that meets another stream there ends the process.

``attention`` is q2d_attention_fwd with q2d_attention_bwd as its gradient.

Options mirror the paper's ablations: ``mode_*`` "rtn" / "sr" choose the
rounding per operand, the "-floor" variants the scale rule that the
truncation-free ablation goes back to; ``activations="1d"`` quantizes X in 1D
blocks (App. C, "Activations"); ``block=64`` uses 64 x 64 blocks (Table 4).
"""
from __future__ import annotations

import itertools
import math

import torch
from torch.autograd.function import once_differentiable

from . import (FP4_1D, FP4_2D, Q2DError, q2d_attention_bwd, q2d_attention_fwd, q2d_gemm, q2d_linear_bwd,
               q2d_linear_fwd, q2d_quantize, q2d_rmsnorm_bwd, q2d_rmsnorm_fwd, q2d_rmsnorm_quantize, QTensor)

_DTYPES = (torch.float32, torch.bfloat16)


class _Q2DLinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, layer):
        K = x.shape[-1]
        if K != weight.shape[1]:
            raise Q2DError("input features %d != weight columns %d" % (K, weight.shape[1]))
        lead = x.shape[:-1]
        dt = x.dtype if x.dtype in _DTYPES else torch.float32
        x2 = x.reshape(-1, K).to(dt).contiguous()
        w = weight.detach().to(dt).contiguous()
        n = layer._calls
        layer._calls += 1
        Y, qX, qW = q2d_linear_fwd(x2, w, layer.mode_x, layer.mode_w, layer.seed, 3 * n, 3 * n + 1,
                                   y_dtype=dt, fmt_x=FP4_1D if layer.activations == "1d" else FP4_2D,
                                   block=layer.block)
        ctx.qX, ctx.qW = qX, qW
        ctx.layer, ctx.offset_dy = layer, 3 * n + 2
        ctx.x_shape, ctx.x_dtype, ctx.w_dtype, ctx.dt = x.shape, x.dtype, weight.dtype, dt
        return Y.reshape(*lead, weight.shape[0])

    @staticmethod
    def backward(ctx, dY):
        layer = ctx.layer
        N = dY.shape[-1]
        dY2 = dY.reshape(-1, N).to(ctx.dt).contiguous()
        dX, dW, _ = q2d_linear_bwd(dY2, ctx.qX, ctx.qW, layer.mode_dy, layer.seed, ctx.offset_dy,
                                   dx_dtype=ctx.dt, dw_dtype=torch.float32, block=layer.block)
        ctx.qX = ctx.qW = None
        return dX.reshape(ctx.x_shape).to(ctx.x_dtype), dW.to(ctx.w_dtype), None


# seeds of layers built without one (distinct per layer within a process)
_SEEDS = itertools.count(0x5EED0001)


class Q2DLinear(torch.nn.Module):
    """Bias-free linear layer on 2D-block FP4 GEMMs (see the module docstring)."""

    def __init__(self, in_features: int, out_features: int, *, mode_x: str = "rtn", mode_w: str = "rtn",
                 mode_dy: str = "sr", activations: str = "2d", block: int = 32, seed: int | None = None,
                 device=None, dtype=torch.float32):
        super().__init__()
        if activations not in ("2d", "1d"):
            raise ValueError("activations must be '2d' or '1d'")
        if seed is None:
            seed = next(_SEEDS)
        self.in_features, self.out_features = in_features, out_features
        self.mode_x, self.mode_w, self.mode_dy = mode_x, mode_w, mode_dy
        self.activations, self.block, self.seed = activations, block, seed
        self.weight = torch.nn.Parameter(torch.empty((out_features, in_features), device=device, dtype=dtype))
        self._calls = 0
        self.reset_parameters()

    def reset_parameters(self):
        torch.nn.init.kaiming_uniform_(self.weight, a=math.sqrt(5))

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return _Q2DLinearFunction.apply(x, self.weight, self)

    def extra_repr(self) -> str:
        return "in=%d, out=%d, x=%s, w=%s, dy=%s, activations=%s, block=%d, seed=%#x" % (
            self.in_features, self.out_features, self.mode_x, self.mode_w, self.mode_dy,
            self.activations, self.block, self.seed)


def _rows(t, cols):
    """t as rows of cols elements that do not share memory, a copy where it has none such."""
    t = t.reshape(-1, cols)
    pitch, one = t.stride()
    return t if (one == 1 or cols == 1) and (pitch >= cols or t.shape[0] < 2) else t.contiguous()


def _kernel_type(t):
    """t in a type that the kernels read (None: none): other ones as float32, as by Q2DLinear."""
    return t if t is None or t.dtype in _DTYPES else t.float()


def _norm_backward(ctx, dy, dh, h, weight, rstd):
    """Gradients of x, the residual and the norm's weight from that of y (None: none) and of h."""
    need_x, need_r, need_w = ctx.needs_input_grad[:3]
    cols = h.shape[1]
    dh = None if dh is None else _rows(dh.to(h.dtype), cols)
    if dy is None:
        # (a copy: dh may be another tensor's gradient too)
        dx, dw = None if dh is None else dh.clone(memory_format=torch.contiguous_format), None
    else:
        dx, dw = q2d_rmsnorm_bwd(dy, h, _kernel_type(weight), rstd, dh=dh, need_dw=need_w)
    if dx is not None:
        # (one object for both where the types agree: as two views of it, either could become its
        # tensor's .grad and share memory with the other's)
        dx = dx.reshape(ctx.x_shape)
    return (dx.to(ctx.x_dtype) if need_x and dx is not None else None,
            dx.to(ctx.r_dtype) if need_r and dx is not None else None,
            None if dw is None else dw.to(weight.dtype))


def _norm_inputs(ctx, x, residual, weight):
    """x and residual as rows."""
    cols = weight.shape[0] if weight.dim() == 1 else -1
    if x.dim() == 0 or x.shape[-1] != cols or (residual is not None and residual.shape != x.shape):
        raise Q2DError("x and residual of one shape [..., %d] are expected" % cols)
    ctx.x_shape, ctx.x_dtype, ctx.r_dtype = x.shape, x.dtype, None if residual is None else residual.dtype
    ctx.set_materialize_grads(False)
    return _rows(x, cols), None if residual is None else _rows(residual, cols)


class _NormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps, y_dtype):
        x2, r2 = _norm_inputs(ctx, x, residual, weight)
        y, h, rstd = q2d_rmsnorm_fwd(x2, weight.detach(), eps, residual=r2, y_dtype=y_dtype)
        ctx.save_for_backward(h, weight, rstd)
        y = y.reshape(x.shape)
        return (y,) if residual is None else (y, h.reshape(x.shape))

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh=None):
        h, weight, rstd = ctx.saved_tensors
        dy = None if dy is None else _rows(dy, h.shape[1])
        return (*_norm_backward(ctx, dy, dh, h, weight.detach(), rstd), None, None)


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5, residual: torch.Tensor | None = None,
             y_dtype=torch.bfloat16):
    """Root-mean-square norm of x [..., cols] times weight [cols], with gradients for all three (once:
    these have none of their own).  With a residual (x's shape) the norm is of h = x + residual
    and (y, h) is returned, otherwise y."""
    out = _NormFunction.apply(x, residual, weight, eps, y_dtype)
    return out[0] if residual is None else out


class _NormLinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, norm_weight, weight, layer, both):
        x2, r2 = (_kernel_type(t) for t in _norm_inputs(ctx, x, residual, norm_weight))
        n = layer._calls
        layer._calls += 1
        both = (True, both and any(ctx.needs_input_grad))
        (qX,), h, rstd = q2d_rmsnorm_quantize(x2, _kernel_type(norm_weight.detach()), layer.eps, residual=r2,
                                              formats=(FP4_1D if layer.activations == "1d" else FP4_2D,),
                                              block=layer.block, orientations=both)
        w = _kernel_type(weight.detach()).contiguous()
        qW = q2d_quantize(w, layer.mode_w, layer.seed, 3 * n + 1, block=layer.block,
                          out=QTensor(FP4_2D, *w.shape, w.device, layer.block, both))
        Y = q2d_gemm(qX, 0, qW, 0, out_dtype=layer.out_dtype)
        ctx.save_for_backward(h, norm_weight, rstd)
        ctx.qX, ctx.qW = qX, qW
        ctx.layer, ctx.offset_dy, ctx.w_dtype = layer, 3 * n + 2, weight.dtype
        Y = Y.reshape(*x.shape[:-1], w.shape[0])
        return (Y,) if residual is None else (Y, h.reshape(x.shape).to(x.dtype))

    @staticmethod
    @once_differentiable
    def backward(ctx, dY, dh=None):
        h, norm_weight, rstd = ctx.saved_tensors
        layer, dy, dW = ctx.layer, None, None
        if dY is not None:
            if ctx.qX is None:
                raise Q2DError("the operands are gone after a backward pass: a second one needs a second forward pass")
            dY2 = _kernel_type(dY.reshape(-1, dY.shape[-1])).contiguous()
            dy, dW, _ = q2d_linear_bwd(dY2, ctx.qX, ctx.qW, layer.mode_dy, layer.seed, ctx.offset_dy, dx_dtype=dY2.dtype,
                                       dw_dtype=torch.float32, block=layer.block)
            dW = dW.to(ctx.w_dtype)
            ctx.qX = ctx.qW = None
        return (*_norm_backward(ctx, dy, dh, h, norm_weight.detach(), rstd), dW, None, None)


class Q2DNormLinear(Q2DLinear):
    """Q2DLinear behind a root-mean-square norm with the residual's addition (see the module
    docstring): y = Q(norm(h) * norm_weight) Q(W)^T with h = x + residual.  X is rounded to
    nearest, with the truncation-free scales.  Inputs and weights of other types than float32 and
    bfloat16 are taken as float32; x + residual and the gradients come back in their own type, Y in
    ``out_dtype``."""

    def __init__(self, in_features: int, out_features: int, *, eps: float = 1e-5, out_dtype=torch.bfloat16, **options):
        if options.get("mode_x", "rtn") != "rtn":
            raise ValueError("the norm's output is rounded to nearest (mode_x 'rtn')")
        super().__init__(in_features, out_features, **options)
        self.eps, self.out_dtype = eps, out_dtype
        self.norm_weight = torch.nn.Parameter(torch.ones(in_features, device=self.weight.device, dtype=self.weight.dtype))

    def reset_parameters(self):
        super().reset_parameters()
        # (Q2DLinear's constructor calls this before there is one)
        if "norm_weight" in self._parameters:
            torch.nn.init.ones_(self.norm_weight)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        """y, or with a residual (y, x + residual)."""
        # (only a backward pass reads the transposed copies)
        out = _NormLinearFunction.apply(x, residual, self.norm_weight, self.weight, self, torch.is_grad_enabled())
        return out[0] if residual is None else out


class _AttentionFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scalars, slopes, documents, prefix):
        out, lse = q2d_attention_fwd(q, k, v, *scalars, slopes, documents, prefix)
        # (the masks too: backward has to meet those of the forward call)
        ctx.save_for_backward(q, k, v, out, lse, slopes, documents, prefix)
        ctx.scalars = scalars
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, *masks = ctx.saved_tensors
        # (a copy of what q2d_attention_bwd does not take; contiguous() keeps an offset)
        *strides, last = dout.stride()
        if last != 1 or any(s % 8 for s in strides) or strides[1] >= 1 << 22 or dout.data_ptr() % 16:
            dout = dout.clone(memory_format=torch.contiguous_format)
        dq, dk, dv = q2d_attention_bwd(dout, q, k, v, out, lse, *ctx.scalars, *masks)
        return dq, dk, dv, None, None, None, None


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float | None = None, causal: bool = True,
              window: int = 0, softcap: float = 0.0, slopes: torch.Tensor | None = None,
              documents: torch.Tensor | None = None, prefix: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of q [batch, len_q, heads_q, dim] on k, v [batch, len_k, heads_kv, dim] with
    gradients for q, k and v (once: these have none of their own); the other arguments as in
    q2d_attention_fwd (slopes get no gradient)."""
    return _AttentionFunction.apply(q, k, v, (scale, causal, window, softcap), slopes, documents, prefix)
