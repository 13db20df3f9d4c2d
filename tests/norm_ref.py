"""Plain 64-bit forms of the norm, its gradient and the clipping of gradients, on the CPU."""
import torch

F32, BF16 = torch.float32, torch.bfloat16


def unit(dtype):
    """Relative error of one rounding."""
    return torch.finfo(dtype).eps / 2


def stream(x, residual):
    """h: the sum in float32, rounded to x's type."""
    x = x.cpu()
    return x if residual is None else (x.float() + residual.cpu().float()).to(x.dtype)


def forward(h, w, eps):
    """rstd [rows, 1] and y in 64 bits, from the rounded h."""
    h = h.double()
    rstd = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    return rstd, h * rstd * w.cpu().double()


def backward(dy, h, w, rstd, dh):
    """dx and dw in 64 bits from a float32 rstd, and what their tolerances are made of."""
    dy, h, w, rstd = dy.cpu().double(), h.cpu().double(), w.cpu().double(), rstd.cpu().double()[:, None]
    dh = torch.zeros_like(h) if dh is None else dh.cpu().double()
    n, g = h * rstd, dy * w
    mean = (g * n).mean(1, keepdim=True)
    dx = rstd * (g - n * mean)
    # float32 steps, u = 2^-24 each: n, g and their product in the mean (3 u of the mean of
    # magnitudes), its rounding (1); n * mean (2 more: n's own and the product's), g (1), their
    # difference, the product with rstd and dh's addition (1 each, of their results)
    u = unit(F32)
    size = (g * n).abs().mean(1, keepdim=True)
    tol = rstd * (n.abs() * (4 * size + 2 * mean.abs()) * u + g.abs() * u) + 2 * u * dx.abs() + u * (dx + dh).abs()
    dw = (dy * n).sum(0)
    # n and the product: 2 u of the sum of magnitudes; the result's rounding
    tol_w = 2 * u * (dy * n).abs().sum(0) + u * dw.abs()
    return dx + dh, tol * (1 + 1e-6), dw, tol_w * (1 + 1e-6)


def clip(tensors, max_norm):
    """The norm in 64 bits, and each tensor times the rounded factor, rounded as defined."""
    norm = torch.sqrt(sum(t.cpu().double().square().sum() for t in tensors))
    f = torch.clamp(max_norm / norm, max=1.0).float()
    return norm, [(t.cpu().float() * f).to(t.dtype) for t in tensors]
