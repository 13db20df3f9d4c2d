"""The norm, its operands and its gradient at the sizes of training: operands in whole tiles (more than 128
of 128 x 256), transposed codes past the cache (48 MB and more), inputs past the cache (above 192 MB)."""
import pytest
import torch

import norm_ref as ref
from helpers import assert_same_bytes, gpu_buffers, poison
from test_gpu_rmsnorm import BF16, DEV, EPS, F32, make, q2d, separate, weight      # noqa: F401

pytestmark = pytest.mark.gpu

FORMATS = [((0,), 32), ((0,), 64), ((2,), 32), ((1,), 32), ((0, 1), 32), ((0, 1), 64), ((2, 1), 32)]
BUFS = ("codes", "codes_t", "scales", "scales_t")


def big(shape, dtype, seed, pad=0):
    """A [rows, cols] view made on the device, rows of different size, `pad` elements apart."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.randn((shape[0], shape[1] + pad), generator=g, device=DEV)
    t *= torch.exp(torch.randn((shape[0], 1), generator=g, device=DEV))
    return t.to(dtype)[:, :shape[1]]


def own_quantizer(q2d, f, y, block):
    return q2d.mxfp8_quantize(y) if f == q2d.MXFP8 else q2d.q2d_quantize_1d(y) if f == q2d.FP4_1D else q2d.q2d_quantize(y, block=block)


# ragged: 1 row and 76 columns, 52 and 132, of the last tile; 170 and 153 tiles
@pytest.mark.parametrize("shape", [(4225, 1100), (2100, 2180)], ids=str)
@pytest.mark.parametrize("formats,block", FORMATS, ids=str)
@pytest.mark.parametrize("x,r,pad", [(BF16, BF16, 0), (BF16, None, 4), (F32, BF16, 0), (F32, None, 1)], ids=str)
def test_operands_in_tiles(q2d, shape, formats, block, x, r, pad):
    """Every byte is that of the quantizer for the float32 y, which the oracle confirms, with blocks
    that are not finite at the edges and in the middle."""
    X, W = make(shape, x, 21, pad), weight(shape[1], F32)
    R = None if r is None else make(shape, r, 22)
    X[shape[0] - 1, 5], X[40, shape[1] - 1], X[2000, 300], W[77] = float("nan"), float("inf"), float("nan"), float("inf")
    y, h, rstd = q2d.q2d_rmsnorm_fwd(X, W, EPS, residual=R, y_dtype=F32)
    out = [q2d.QTensor(f, *shape, DEV, block if f == q2d.FP4_2D else 32) for f in formats]
    for q in out:
        poison(q)
    print(shape, formats, block, x, r, pad, flush=True)
    qs, h2, rstd2 = q2d.q2d_rmsnorm_quantize(X, W, EPS, residual=R, formats=formats, out=out)
    assert qs is out and torch.equal(rstd.nan_to_num(-1), rstd2.nan_to_num(-1))
    for q, f in zip(qs, formats):
        own, want = separate(q2d, f, y, block)
        assert_same_bytes(gpu_buffers(q), own, "quantizer, format %d" % f)
        assert_same_bytes(gpu_buffers(q), want, "oracle, format %d" % f)
    for orientations in ((True, False), (False, True)):
        one, _, _ = q2d.q2d_rmsnorm_quantize(X, W, EPS, residual=R, formats=formats, block=block, orientations=orientations)
        for a, b in zip(qs, one):
            got = gpu_buffers(b)
            assert set(got) == ({"codes", "scales"} if orientations[0] else {"codes_t", "scales_t"})
            assert_same_bytes(got, {k: v for k, v in gpu_buffers(a).items() if k in got})


# transposed codes of 50.4 MB each
@pytest.mark.parametrize("shape,formats,block", [((8200, 4100), (0, 1), 32), ((8200, 4100), (0, 1), 64), ((8200, 4100), (2, 1), 32),
                                                 ((8200, 6150), (1,), 32), ((16400, 6150), (0,), 32), ((16400, 6150), (0,), 64),
                                                 ((16400, 6150), (2,), 32)], ids=str)
@pytest.mark.parametrize("dtype,pad", [(BF16, 0), (F32, 2)], ids=str)
def test_operands_past_the_cache(q2d, shape, formats, block, dtype, pad):
    X, W = big(shape, dtype, 23, pad), weight(shape[1], BF16)
    X[5, 5], X[shape[0] - 1, shape[1] - 1] = float("nan"), float("inf")
    y = q2d.q2d_rmsnorm_fwd(X, W, EPS, y_dtype=F32)[0]
    out = [q2d.QTensor(f, *shape, DEV, block if f == q2d.FP4_2D else 32) for f in formats]
    for q in out:
        poison(q)
    print(shape, formats, block, dtype, pad, flush=True)
    q2d.q2d_rmsnorm_quantize(X, W, EPS, formats=formats, out=out)
    for q, f in zip(out, formats):
        own = own_quantizer(q2d, f, y, block)
        for k in BUFS:
            assert torch.equal(getattr(q, k), getattr(own, k)), (f, k)


# a width for each split of a row's work
WIDTHS = [200, 1000, 2049, 4096, 5001, 8000, 12289, 17000]
MB = 1 << 20


def rows_for(cols, bytes_each):
    """Rows that take the inputs above 192 MB, and an odd number of them."""
    return (193 * MB // (cols * bytes_each)) | 1


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("x,r,y", [(BF16, BF16, BF16), (F32, BF16, F32), (BF16, F32, BF16), (F32, None, BF16)], ids=str)
def test_forward_past_the_cache(q2d, cols, x, r, y):
    """A row's results do not depend on how many rows there are."""
    size = (2 if x == BF16 else 4) + (0 if r is None else 2 if r == BF16 else 4)
    shape = (rows_for(cols, size), cols)
    X, R, W = big(shape, x, 31, 3), None if r is None else big(shape, r, 32, 1), weight(cols, F32)
    print(shape, x, r, y, flush=True)
    Y, H, S = q2d.q2d_rmsnorm_fwd(X, W, EPS, residual=R, y_dtype=y)
    third = shape[0] // 3 + 1
    for a in range(0, shape[0], third):
        part = slice(a, a + third)
        y1, h1, s1 = q2d.q2d_rmsnorm_fwd(X[part], W, EPS, residual=None if R is None else R[part], y_dtype=y)
        assert torch.equal(Y[part], y1) and torch.equal(H[part], h1) and torch.equal(S[part], s1), a
    # a few rows against 64 bits
    some = torch.arange(0, shape[0], max(1, shape[0] // 7), device=DEV)
    want, yy = ref.forward(ref.stream(X[some], None if R is None else R[some]), W, EPS)
    u = ref.unit(F32)
    assert float(((S[some].cpu().double()[:, None] - want).abs() / want).max()) <= u * (1 + 1e-9)
    lim = yy.abs() * (3 * u + (ref.unit(y) if y == BF16 else 0)) * 1.00001
    assert bool(((Y[some].cpu().double() - yy).abs() <= lim + 1e-44).all())


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("x,y", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)], ids=str)
@pytest.mark.parametrize("residual", [True, False])
def test_backward_past_the_cache(q2d, cols, x, y, residual):
    size = (2 if x == BF16 else 4) * (2 if residual else 1) + (2 if y == BF16 else 4)
    shape = (rows_for(cols, size), cols)
    H, dY, dH = big(shape, x, 41, 1), big(shape, y, 42, 3) * 1e-3, big(shape, x, 43) * 1e-3 if residual else None
    W = weight(cols, F32)
    S = q2d.q2d_rmsnorm_fwd(H, W, EPS)[2]
    print(shape, x, y, residual, flush=True)
    dx, dw = q2d.q2d_rmsnorm_bwd(dY, H, W, S, dh=dH)
    third = shape[0] // 3 + 1
    for a in range(0, shape[0], third):
        part = slice(a, a + third)
        d1, _ = q2d.q2d_rmsnorm_bwd(dY[part], H[part], W, S[part], dh=None if dH is None else dH[part])
        assert torch.equal(dx[part], d1), a
    # the weights' gradient: n rounds once, a workgroup's part once, and the result; products and sums are
    # in 64 bits
    want, size = torch.zeros(cols, dtype=torch.float64, device=DEV), torch.zeros(cols, dtype=torch.float64, device=DEV)
    for a in range(0, shape[0], 4096):
        part = slice(a, a + 4096)
        p = dY[part].double() * (H[part].double() * S[part].double()[:, None])
        want += p.sum(0)
        size += p.abs().sum(0)
    u = ref.unit(F32)
    assert bool(((dw.double() - want).abs() <= (2 * u * size + u * want.abs()) * (1 + 1e-6) + 1e-44).all())
