"""The operators around the quantized linear layers as timed cases: the root-mean-square norm
with the residual's addition, whose output may be a GEMM operand in 4 or 8 bits, its gradient,
and the gradients' global norm with clipping.

Kinds of case, each one pass through the public entry points:

  norm      q2d_rmsnorm_fwd: h = x + residual, y = norm(h) * weight in float32 or bfloat16
  quantize  q2d_rmsnorm_quantize: the same with y as quantized operands (2D or 1D FP4, MXFP8),
            then q2d_dequantize of every stored copy: the values that the GEMMs multiply
  train     q2d_rmsnorm_fwd, then q2d_rmsnorm_bwd with the gradient that comes through the
            residual stream; outputs and gradients
  total     q2d_grad_norm: the 2-norm over all elements of many tensors
  clip      q2d_clip_grads: that norm, and the tensors scaled where it is above max_norm

h is rounded to the type of x, and the norm is of the rounded h.  rstd = 1 / sqrt(mean(h^2) +
eps) rounds to 32 bits once, y is (h * rstd) * weight with both products rounded to 32 bits;
operands hold the codes of that y, rounded to nearest:

  2d     E2M1 codes, one power of two for each 32 x 32 (or 64 x 64) block, both copies alike
  1d     E2M1 codes, 1 x 32 blocks in the rowwise copy, 32 x 1 blocks in the other
  mx     E4M3 codes, blocks as 1d

with the smallest power of two for which a block's largest magnitude does not pass the
format's largest value.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-5


# ---------------------------------------------------------------- the cases

def _matrices(*shapes, times=1):
    return ",".join(",".join("%dx%d" % s for s in shapes) for _ in range(times))


def listed():
    return [
        # one decoded token of a 7B-class model, residual stream in bfloat16: latency
        dict(name="norm_token", kind="norm", rows=1, cols=4096, x="bf16", r="bf16", w="bf16", y="bf16", pitch=0),
        # evaluation of whole sequences, hidden 4096: a float32 stream and a layer's bfloat16 output
        dict(name="norm_7b", kind="norm", rows=16384, cols=4096, x="f32", r="bf16", w="f32", y="bf16", pitch=0),
        # nothing a multiple of anything: rows of a wider float32 tensor, no residual
        dict(name="norm_odd_f32", kind="norm", rows=1999, cols=1111, x="f32", r="", w="f32", y="f32", pitch=5),
        # the Tiny configuration in training, float32: launches and host calls count
        dict(name="quantize_tiny", kind="quantize", rows=128, cols=256, x="f32", r="bf16", w="f32", formats="2d",
             both=True, pitch=0),
        # 64 sequences that decode: operands of the query/key and of the value projection, rowwise copies only
        dict(name="quantize_decode_64", kind="quantize", rows=64, cols=4096, x="bf16", r="bf16", w="bf16",
             formats="2d,mx", both=False, pitch=0),
        # a training step of the 7B-class block: MXFP8 for query and key, FP4 for the value projection
        dict(name="quantize_7b_mixed", kind="quantize", rows=16384, cols=4096, x="bf16", r="bf16", w="f32",
             formats="2d,mx", both=True, pitch=0),
        # the 1B-class MLP's input in the paper's activation placement (1D blocks), float32 stream
        dict(name="quantize_1b_1d", kind="quantize", rows=8192, cols=2048, x="f32", r="bf16", w="f32", formats="1d",
             both=True, pitch=0),
        # training of the 7B-class block's norm, bfloat16 stream
        dict(name="train_7b", kind="train", rows=16384, cols=4096, x="bf16", r="bf16", w="f32", y="bf16", pitch=0),
        # a ragged micro-batch, odd width, float32 stream
        dict(name="train_odd", kind="train", rows=777, cols=2049, x="f32", r="bf16", w="f32", y="bf16", pitch=0),
        # gradients of the Tiny configuration's layers
        dict(name="total_tiny", kind="total", tensors=_matrices((768, 256), (256, 256), (1, 256), (1024, 256),
                                                                (256, 1024), (1, 256)), dtype="f32", scale=1e-3),
        # gradients of a model of many small layers in bfloat16, ragged sizes: 240 tensors
        dict(name="clip_many", kind="clip", tensors=_matrices((1536, 512), (512, 512), (512, 1), (1365, 512), (512, 1365),
                                                              (513, 1), times=40), dtype="bf16", scale=1e-3,
             max_norm=1.0),
        # float32 gradients of two 7B-class blocks, clipped
        dict(name="clip_7b", kind="clip", tensors=_matrices((12288, 4096), (4096, 4096), (4096, 1), (11008, 4096),
                                                            (11008, 4096), (4096, 11008), (4096, 1), times=2),
             dtype="f32", scale=1e-3, max_norm=1.0),
    ]


def _log(rng, lo, hi, step=1):
    """Log-uniform in [lo, hi], rounded to a multiple of step."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, min(hi, int(round(v / step)) * step))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["norm", "norm", "quantize", "quantize", "quantize", "train", "train", "total", "clip", "clip"])
    types = ["bf16", "bf16", "f32"]
    if kind in ("total", "clip"):
        dtype, most = rng.choice(types), 400e6
        sizes, total = [], 0
        largest = _log(rng, 64, 12288)
        for _ in range(_log(rng, 1, 400)):
            s = (_log(rng, 1, largest), _log(rng, 1, largest))
            if total + s[0] * s[1] > most:
                break
            sizes.append(s)
            total += s[0] * s[1]
        sizes = sizes or [(largest, 7)]
        c = dict(kind=kind, tensors=_matrices(*sizes), dtype=dtype, scale=10.0 ** rng.uniform(-6, 0))
        if kind == "clip":
            c["max_norm"] = rng.choice([0.5, 1.0, 1.0, 1e6])
        return c
    while True:
        rows, cols = _log(rng, 1, 16384), _log(rng, 64, 12288, rng.choice([64, 64, 64, 8, 1]))
        x = rng.choice(types)
        if rows * cols * (2 if x == "f32" else 1) <= 0.9 * 16384 * 4096:
            break
    c = dict(kind=kind, rows=rows, cols=cols, x=x, r=rng.choice(["", "bf16", "bf16", x]), w=rng.choice(["f32", "f32", "bf16"]),
             pitch=rng.choice([0, 0, 0, 1, 8, 100]))
    if kind == "quantize":
        c.update(formats=rng.choice(["2d", "2d", "2d64", "1d", "mx", "2d,mx", "1d,mx"]), both=rng.random() < 0.7)
    else:
        c["y"] = rng.choice(types)
    return c


# ---------------------------------------------------------------- sizes and work

_BYTES = {"f32": 4, "bf16": 2, "": 0}
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _shapes(c):
    return [tuple(int(n) for n in s.split("x")) for s in c["tensors"].split(",")]


def work(case):
    c = case
    if c["kind"] in ("total", "clip"):
        n = sum(a * b for a, b in _shapes(c))
        return {"bytes": n * _BYTES[c["dtype"]] * (1 if c["kind"] == "total" else 2),
                "flops": n * (2 if c["kind"] == "total" else 3)}
    n, e = c["rows"] * c["cols"], _BYTES[c["x"]]
    # x and residual read, h written (x itself where there is no residual)
    stream = n * (e + _BYTES[c["r"]] + (e if c["r"] else 0)) + 4 * c["rows"]
    if c["kind"] == "norm":
        return {"bytes": stream + n * _BYTES[c["y"]], "flops": 5 * n}
    if c["kind"] == "train":
        # dy, h and dh read, dx written
        return {"bytes": stream + n * _BYTES[c["y"]] * 2 + 3 * n * e, "flops": 15 * n}
    # each copy's codes written, read back, and its values written in 16 bits
    copies = 2 if c["both"] else 1
    codes = sum(1.0 if f == "mx" else 0.5 for f in c["formats"].split(","))
    return {"bytes": stream + n * copies * (2 * codes + 2 * len(c["formats"].split(","))), "flops": 8 * n}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _stream(c, g, dtype):
    """A residual stream: rows of different size, some channels far larger than the others."""
    x = torch.randn((c["rows"], c["cols"] + c["pitch"]), generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn((c["rows"], 1), generator=g, device=DEV))
    channels = torch.rand((1, c["cols"] + c["pitch"]), generator=g, device=DEV)
    x *= torch.where(channels < 0.01, 20.0, 1.0)
    return x.to(_TYPES[dtype])[:, :c["cols"]]


def prepare(case, seed):
    c, g = case, _generator(seed)
    if c["kind"] in ("total", "clip"):
        dt = _TYPES[c["dtype"]]
        st = {"case": c, "grads": [torch.randn(s, generator=g, device=DEV).mul_(c["scale"]).to(dt) for s in _shapes(c)]}
        if c["kind"] == "clip":
            # the clipped gradients lie one behind the other in one buffer, as a bucket for communication does
            sizes = [t.numel() for t in st["grads"]]
            st["flat"] = torch.empty(sum(sizes), dtype=dt, device=DEV)
            st["out"] = [o.view(t.shape) for o, t in zip(st["flat"].split(sizes), st["grads"])]
        return st
    R, C = c["rows"], c["cols"]
    st = {"case": c, "x": _stream(c, g, c["x"]),
          "r": torch.randn((R, C), generator=g, device=DEV).to(_TYPES[c["r"]]) if c["r"] else None,
          "w": (1 + 0.2 * torch.randn(C, generator=g, device=DEV)).to(_TYPES[c["w"]])}
    if c["kind"] == "train":
        st["dy"] = (1e-3 * torch.randn((R, C), generator=g, device=DEV)).to(_TYPES[c["y"]])
        st["dh"] = (1e-3 * torch.randn((R, C), generator=g, device=DEV)).to(_TYPES[c["x"]])
    return st


# ---------------------------------------------------------------- the plain forms

def _plain_norm(st):
    """h, rstd [rows, 1] and y in 32 bits."""
    x, r = st["x"], st["r"]
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    # (64 bits for the sum: codes next to a border hang on the last bit)
    mean = h.double().square().sum(dim=1, keepdim=True) / h.shape[1]
    rstd = (1.0 / torch.sqrt(mean + EPS)).float()
    return h, rstd, (h.float() * rstd) * st["w"].float()


def _e2m1(v):
    """Magnitudes in [0, 6] to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    step = torch.where(v < 2, 0.5, torch.where(v < 4, 1.0, 2.0))
    return torch.round(v / step) * step


def _plain_blocks(y, fmt, bh, bw):
    """Values of y in blocks of bh x bw, in 16 bits (exact: the codes have few digits)."""
    R, C = y.shape
    p = torch.nn.functional.pad(y, (0, -C % bw, 0, -R % bh)).view(-(-R // bh), bh, -(-C // bw), bw)
    top, bits = (448.0, 9) if fmt == "mx" else (6.0, 3)
    m, e = torch.frexp(p.abs().amax(dim=(1, 3), keepdim=True))
    # largest value = 0.875 * 2^9 or 0.75 * 2^3
    e = torch.where(m > 0, e - bits + (m > top / 2 ** bits).to(e.dtype), torch.full_like(e, -127)).clamp(min=-127)
    v = torch.ldexp(p, -e)
    v = v.to(torch.float8_e4m3fn).float() if fmt == "mx" else torch.copysign(_e2m1(v.abs()), v)
    return torch.ldexp(v, e).view(R + -R % bh, C + -C % bw)[:R, :C].to(torch.bfloat16)


def _edges(fmt):
    return {"2d": ((32, 32), (32, 32)), "2d64": ((64, 64), (64, 64))}.get(fmt, ((1, 32), (32, 1)))


def _plain(st):
    c = st["case"]
    if c["kind"] in ("total", "clip"):
        norm = torch.stack([t.double().square().sum() for t in st["grads"]]).sum().sqrt()
        if c["kind"] == "total":
            return norm.float()
        scale = (c["max_norm"] / norm).clamp(max=1.0).float()
        return [norm.float(), torch.cat([(t.float() * scale).to(t.dtype).flatten() for t in st["grads"]])]
    h, rstd, y = _plain_norm(st)
    if c["kind"] == "quantize":
        return [h, rstd.view(-1)] + [_plain_blocks(y, f, *_edges(f)[k])
                                     for f in c["formats"].split(",") for k in range(2 if c["both"] else 1)]
    out = [y.to(_TYPES[c["y"]]), h, rstd.view(-1)]
    if c["kind"] == "norm":
        return out
    dy, w = st["dy"].float(), st["w"].float()
    xh, g = h.float() * rstd, dy * w
    dx = rstd * (g - xh * (g * xh).mean(dim=1, keepdim=True)) + st["dh"].float()
    return out + [dx.to(h.dtype), (dy * xh).sum(dim=0)]


# ---------------------------------------------------------------- one pass

def run(state):
    if not own:
        return _plain(state)
    import paper_2607_24953_amd as q2d
    st, c = state, state["case"]
    if c["kind"] == "total":
        return q2d.q2d_grad_norm(st["grads"])
    if c["kind"] == "clip":
        return [q2d.q2d_clip_grads(st["grads"], c["max_norm"], out=st["out"]), st["flat"]]
    if c["kind"] == "quantize":
        formats = {"2d": q2d.FP4_2D, "2d64": q2d.FP4_2D, "1d": q2d.FP4_1D, "mx": q2d.MXFP8}
        qs, h, rstd = q2d.q2d_rmsnorm_quantize(st["x"], st["w"], EPS, residual=st["r"],
                                               formats=tuple(formats[f] for f in c["formats"].split(",")),
                                               block=64 if c["formats"] == "2d64" else 32, orientations=(True, c["both"]))
        return [h, rstd] + [q2d.q2d_dequantize(q, k, torch.bfloat16) for q in qs for k in range(2 if c["both"] else 1)]
    y, h, rstd = q2d.q2d_rmsnorm_fwd(st["x"], st["w"], EPS, residual=st["r"], y_dtype=_TYPES[c["y"]])
    if c["kind"] == "norm":
        return [y, h, rstd]
    return [y, h, rstd, *q2d.q2d_rmsnorm_bwd(st["dy"], h, st["w"], rstd, dh=st["dh"])]


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_blocks(y, fmt, bh, bw):
    """y's values by the format's table, one block row at a time."""
    if fmt == "mx":
        table = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
        table = table[:-1]                                  # (the last code is NaN)
    else:
        table = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    grid = torch.tensor(table, dtype=torch.float64, device=y.device)
    middle = (grid[1:] + grid[:-1]) / 2
    odd = torch.arange(len(table) - 1, device=y.device) % 2 == 1    # a tie below an even code goes up
    middle = torch.where(odd, middle, torch.nextafter(middle, torch.full_like(middle, 1e9)))
    out = torch.empty_like(y)
    R, C = y.shape
    step = max(bh, (1 << 24) // C // bh * bh)
    for r in range(0, R, step):
        v = y[r:r + step]
        n = v.shape[0]
        top = torch.nn.functional.pad(v.abs(), (0, -C % bw, 0, -n % bh))
        top = top.unflatten(0, (-1, bh)).unflatten(2, (-1, bw)).amax(dim=3).amax(dim=1)
        s = torch.exp2(torch.ceil(torch.log2((top / grid[-1]).clamp(min=2.0 ** -127))))
        s = torch.where(s * grid[-1] < top, 2 * s, torch.where(s / 2 * grid[-1] >= top, s / 2, s)).clamp(min=2.0 ** -127)
        s = s.repeat_interleave(bh, dim=0)[:n].repeat_interleave(bw, dim=1)[:, :C]
        out[r:r + step] = torch.sign(v) * grid[torch.bucketize(v.abs() / s, middle, right=True)] * s
    return out


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["kind"] in ("total", "clip"):
        norm = math.sqrt(math.fsum(float(torch.dot(t.double().flatten(), t.double().flatten())) for t in st["grads"]))
        total = np.float64(norm)
        if c["kind"] == "total":
            return total
        return [total, torch.cat([t.flatten() for t in st["grads"]]).double() * min(1.0, c["max_norm"] / norm)]
    h, w = st["x"].double(), st["w"].double()
    if st["r"] is not None:
        h = (h + st["r"].double()).to(st["x"].dtype).double()      # (the stream's type is part of the definition)
    length = torch.linalg.vector_norm(h, dim=1, keepdim=True)
    rstd = (length * length / c["cols"] + EPS) ** -0.5
    n = h * rstd
    if c["kind"] == "quantize":
        return [h, rstd[:, 0]] + [_exact_blocks(n * w, f, *_edges(f)[k])
                                  for f in c["formats"].split(",") for k in range(2 if c["both"] else 1)]
    out = [n * w, h, rstd[:, 0]]
    if c["kind"] == "norm":
        return out
    dy = st["dy"].double()
    along = torch.linalg.vecdot(dy * w, n, dim=1)[:, None] / c["cols"]
    return out + [(dy * w - along * n) * rstd + st["dh"].double(), torch.linalg.vecdot(dy, n, dim=0)]
