"""The root-mean-square norm against 64 bits: values, statistics, quantized operands, gradient."""
import pytest
import torch

import norm_ref as ref
import oracle
from helpers import assert_same_bytes, gpu_buffers, poison

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5
# rows x columns: single rows and elements, widths around the vector loads and the work splits of a
# row, long rows, many short ones
SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (64, 72), (33, 100), (130, 257), (7, 1024), (9, 2048), (2, 2050), (65, 4096),
          (3, 4104), (2, 8192), (2, 11008), (3, 16384), (2, 16392), (2, 32768), (2, 40001), (1, 100003), (5000, 64), (2100, 33)]


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def make(shape, dtype, seed, pad=0, shift=0):
    """A [rows, cols] view whose rows lie `pad` elements apart, `shift` elements into its memory."""
    g = torch.Generator().manual_seed(seed)
    rows, cols = shape
    t = torch.randn((rows, cols), generator=g) * torch.exp(torch.randn((rows, 1), generator=g))
    buf = torch.full((rows * (cols + pad) + shift,), 7.0, dtype=dtype, device=DEV)
    view = buf[shift:].view(rows, cols + pad)[:, :cols]
    view.copy_(t.to(dtype))
    return view


def weight(cols, dtype, seed=5):
    return (1 + 0.2 * torch.randn(cols, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)


def check_forward(y, h, rstd, x, r, w, eps=EPS):
    want = ref.stream(x, r)
    assert torch.equal(h.cpu(), want)
    rs, yy = ref.forward(want, w, eps)
    u = ref.unit(F32)
    assert float(((rstd.cpu().double()[:, None] - rs).abs() / rs).max()) <= u * (1 + 1e-9)
    # rstd, two products, the output's rounding
    lim = yy.abs() * (3 * u + (ref.unit(y.dtype) if y.dtype == BF16 else 0)) * 1.00001
    assert bool(((y.cpu().double() - yy).abs() <= lim + 1e-44).all())


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("x,r,w,y", [(BF16, BF16, BF16, BF16), (F32, BF16, F32, BF16), (F32, None, F32, F32), (BF16, F32, F32, F32)], ids=str)
def test_forward(q2d, shape, x, r, w, y):
    X, R, W = make(shape, x, 1), None if r is None else make(shape, r, 2), weight(shape[1], w)
    check_forward(*q2d.q2d_rmsnorm_fwd(X, W, EPS, residual=R, y_dtype=y), X, R, W)


@pytest.mark.parametrize("cols", [8, 100, 1000, 4096, 20000, 33000])
@pytest.mark.parametrize("pads", [(1, 0, 3, 2), (8, 8, 8, 8), (0, 5, 0, 0)], ids=str)
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_forward_rows_anywhere(q2d, cols, pads, shift):
    """Rows of any pitch and alignment, outputs too; what lies between rows is left alone."""
    shape = (5, cols)
    for x, r in ((BF16, F32), (F32, BF16), (F32, None)):
        X, R = make(shape, x, 3, pads[0], shift), None if r is None else make(shape, r, 4, pads[1], shift)
        h, y = None if r is None else make(shape, x, 5, pads[2], shift), make(shape, BF16, 6, pads[3], shift)
        out = q2d.q2d_rmsnorm_fwd(X, weight(cols, F32), EPS, residual=R, h=h, y=y)
        assert out[0] is y and (r is None or out[1] is h)
        check_forward(*out, X, R, weight(cols, F32))
        for t, pad in ((y, pads[3]), (h, pads[2])):
            if t is not None and pad:
                wide = torch.as_strided(t, (4, pad), (cols + pad, 1), t.storage_offset() + cols)
                assert bool((wide == 7).all())


def test_forward_in_place(q2d):
    for dt, shape in ((BF16, (70, 4096)), (F32, (70, 1001)), (BF16, (3, 50000))):
        X, R, W = make(shape, dt, 8), make(shape, dt, 9), weight(shape[1], F32)
        y, h, rstd = q2d.q2d_rmsnorm_fwd(X, W, EPS, residual=R)
        for place in ("x", "r"):
            x2, r2 = X.clone(), R.clone()
            at = x2 if place == "x" else r2
            got = q2d.q2d_rmsnorm_fwd(x2, W, EPS, residual=r2, h=at)
            assert got[1] is at and torch.equal(at, h) and torch.equal(got[0], y) and torch.equal(got[2], rstd)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-20, 1e20, 1e36])
def test_any_size(q2d, scale):
    """Squares that leave float32's range: the statistics do not."""
    X = (make((9, 513), F32, 11).sign() * (1 + torch.rand((9, 513), device=DEV))) * scale
    y, h, rstd = q2d.q2d_rmsnorm_fwd(X, weight(513, F32), 1e-30, y_dtype=F32)
    rs, yy = ref.forward(X.cpu(), weight(513, F32), 1e-30)
    # (a rstd below 2^-126 has a step of 2^-149)
    err = (rstd.cpu().double()[:, None] - rs).abs()
    assert bool((err <= rs * 2.0 ** -24 * (1 + 1e-9) + 2.0 ** -150).all())
    lim = yy.abs() * (2.0 ** -22 + 2.0 ** -150 / rs)
    assert bool(((y.cpu().double() - yy).abs() <= lim + 1e-44).all())


def test_zero_rows_and_rows_of_zeros(q2d):
    W = weight(300, F32)
    y, h, rstd = q2d.q2d_rmsnorm_fwd(torch.zeros((0, 300), device=DEV), W)
    assert y.shape == (0, 300) and rstd.shape == (0,)
    dx, dw = q2d.q2d_rmsnorm_bwd(y, torch.zeros((0, 300), device=DEV), W, rstd)
    assert dx.shape == (0, 300) and torch.equal(dw, torch.zeros_like(dw))
    y, h, rstd = q2d.q2d_rmsnorm_fwd(torch.zeros((4, 300), device=DEV), W)
    assert float(y.abs().max()) == 0 and bool((rstd == torch.tensor(1e-5, dtype=torch.float64).rsqrt().float().item()).all())


def test_not_finite(q2d):
    """A row's NaN or infinity stays in its row, and follows the formula there."""
    X, W = make((6, 700), F32, 12), weight(700, F32)
    X[1, 699], X[3, 0], X[4, 5] = float("nan"), float("inf"), -float("inf")
    y, h, rstd = q2d.q2d_rmsnorm_fwd(X, W, y_dtype=F32)
    good = [0, 2, 5]
    check_forward(y[good], h[good], rstd[good], X[good], None, W)
    assert bool(y[1].isnan().all()) and float(rstd[3]) == 0 and float(rstd[4]) == 0
    for row, col in ((3, 0), (4, 5)):
        bad = y[row].isnan()
        assert bool(bad[col]) and int(bad.sum()) == 1 and float(y[row][~bad].abs().max()) == 0


def test_far_rows(q2d):
    """Offsets that pass 2^32 bytes and 2^31 elements."""
    pitch = (1 << 30) + 8
    buf = torch.empty(2 * pitch + 4096, dtype=BF16, device=DEV)
    X = torch.as_strided(buf, (3, 4096), (pitch, 1))
    X.copy_(make((3, 4096), BF16, 14))
    W = weight(4096, F32)
    check_forward(*q2d.q2d_rmsnorm_fwd(X, W), X, None, W)
    q, _, _ = q2d.q2d_rmsnorm_quantize(X, W)
    q2, _, _ = q2d.q2d_rmsnorm_quantize(X.clone(), W)
    assert_same_bytes(gpu_buffers(q[0]), {k: v for k, v in gpu_buffers(q2[0]).items()})
    dy = torch.as_strided(torch.empty(2 * pitch + 4096, dtype=BF16, device=DEV), (3, 4096), (pitch, 1))
    dy.copy_(make((3, 4096), BF16, 15))
    rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
    far = q2d.q2d_rmsnorm_bwd(dy, X, W, rstd)
    near = q2d.q2d_rmsnorm_bwd(dy.clone(), X.clone(), W, rstd)
    assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])


# ---------------------------------------------------------------- operands

QSHAPES = [(1, 1), (1, 4096), (3, 7), (31, 8), (64, 200), (100, 129), (128, 256), (129, 257), (257, 1000), (40, 4100), (300, 2048),
           (2000, 72), (5, 12288)]


def separate(q2d, f, y, block):
    """The library's own quantizer for the float32 y; and the oracle's bytes."""
    c = y.cpu()
    if f == q2d.MXFP8:
        return gpu_buffers(q2d.mxfp8_quantize(y)), oracle.quantize_mxfp8(c)
    if f == q2d.FP4_1D:
        return gpu_buffers(q2d.q2d_quantize_1d(y)), oracle.quantize_fp4_1d(c)
    return gpu_buffers(q2d.q2d_quantize(y, block=block)), oracle.quantize_fp4_2d(c, block=block)


@pytest.mark.parametrize("shape", QSHAPES, ids=str)
@pytest.mark.parametrize("formats,block", [((0,), 32), ((0,), 64), ((2,), 32), ((1,), 32), ((0, 1), 32), ((1, 2), 32)], ids=str)
@pytest.mark.parametrize("x,r,w", [(BF16, BF16, F32), (F32, BF16, BF16), (F32, None, F32)], ids=str)
def test_operands(q2d, shape, formats, block, x, r, w):
    """Every byte is that of the quantizer for the float32 y, and of the oracle."""
    X, R, W = make(shape, x, 21), None if r is None else make(shape, r, 22), weight(shape[1], w)
    y, h, rstd = q2d.q2d_rmsnorm_fwd(X, W, EPS, residual=R, y_dtype=F32)
    out = [q2d.QTensor(f, *shape, DEV, block if f == q2d.FP4_2D else 32) for f in formats]
    for q in out:
        poison(q)
    qs, h2, rstd2 = q2d.q2d_rmsnorm_quantize(X, W, EPS, residual=R, formats=formats, out=out)
    assert qs is out and torch.equal(h, h2) and torch.equal(rstd, rstd2)
    for q, f in zip(qs, formats):
        own, want = separate(q2d, f, y, block)
        assert_same_bytes(gpu_buffers(q), own, "quantizer, format %d" % f)
        assert_same_bytes(gpu_buffers(q), want, "oracle, format %d" % f)


@pytest.mark.parametrize("formats", [(0,), (2,), (1,), (0, 1)], ids=str)
@pytest.mark.parametrize("shape,pad,shift", [((130, 1000), 3, 1), ((70, 70), 0, 2), ((33, 4096), 8, 0), ((17, 5), 1, 3)], ids=str)
def test_operands_of_rows_anywhere(q2d, formats, shape, pad, shift):
    for dt in (BF16, F32):
        X, W = make(shape, dt, 23, pad, shift), weight(shape[1], F32)
        y = q2d.q2d_rmsnorm_fwd(X, W, y_dtype=F32)[0]
        qs, _, _ = q2d.q2d_rmsnorm_quantize(X, W, formats=formats)
        for q, f in zip(qs, formats):
            assert_same_bytes(gpu_buffers(q), separate(q2d, f, y, 32)[0], "format %d" % f)


@pytest.mark.parametrize("formats", [(0,), (2,), (1,), (0, 1), (2, 1)], ids=str)
@pytest.mark.parametrize("orientations", [(True, False), (False, True)], ids=str)
@pytest.mark.parametrize("rows", [1, 20, 200])
def test_one_orientation(q2d, formats, orientations, rows):
    X, R, W = make((rows, 520), BF16, 24), make((rows, 520), BF16, 25), weight(520, F32)
    both, h, _ = q2d.q2d_rmsnorm_quantize(X, W, residual=R, formats=formats)
    one, h2, _ = q2d.q2d_rmsnorm_quantize(X, W, residual=R, formats=formats, orientations=orientations)
    assert torch.equal(h, h2)
    for a, b in zip(both, one):
        got = gpu_buffers(b)
        assert set(got) == ({"codes", "scales"} if orientations[0] else {"codes_t", "scales_t"})
        assert_same_bytes(got, {k: v for k, v in gpu_buffers(a).items() if k in got})


@pytest.mark.parametrize("formats", [(0,), (2,), (1,), (0, 1)], ids=str)
@pytest.mark.parametrize("rows", [3, 70])
def test_operands_not_finite(q2d, formats, rows):
    """Blocks with a NaN or an infinity, at the matrix's edge too, and a weight that is not finite."""
    shape = (rows, 77)
    for where in ("x", "w"):
        X, W = make(shape, F32, 26), weight(77, F32)
        if where == "x":
            X[rows - 1, 76], X[0, 33], X[1, 2] = float("nan"), float("inf"), float("nan")
        else:
            W[76], W[40] = float("inf"), float("nan")
        y = q2d.q2d_rmsnorm_fwd(X, W, y_dtype=F32)[0]
        qs, _, _ = q2d.q2d_rmsnorm_quantize(X, W, formats=formats)
        for q, f in zip(qs, formats):
            own, want = separate(q2d, f, y, 32)
            assert_same_bytes(gpu_buffers(q), own)
            assert_same_bytes(gpu_buffers(q), want)


def test_values_beside_operands(q2d):
    """The C entry point writes values and operands in one call."""
    import ctypes
    from paper_2607_24953_amd import norms as N
    X, R, W = make((70, 300), BF16, 27), make((70, 300), BF16, 28), weight(300, F32)
    want, h, rstd = q2d.q2d_rmsnorm_quantize(X, W, EPS, residual=R, formats=(0, 1))
    y = q2d.q2d_rmsnorm_fwd(X, W, EPS, residual=R, y_dtype=F32)[0]
    qs, y2, h2, rstd2 = [q2d.QTensor(f, 70, 300, DEV) for f in (0, 1)], torch.zeros_like(y), torch.zeros_like(h), torch.zeros_like(rstd)
    n = N._Norm(x_dtype=1, residual_dtype=1, weight_dtype=0, y_dtype=0, rows=70, cols=300, eps=EPS, x=X.data_ptr(), ldx=300,
                residual=R.data_ptr(), ld_residual=300, weight=W.data_ptr(), h=h2.data_ptr(), ldh=300, y=y2.data_ptr(), ldy=300,
                rstd=rstd2.data_ptr())
    assert q2d._lib.q2d_rmsnorm_fwd(ctypes.byref(n), qs[0].ptr(), qs[1].ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(rstd, rstd2)
    for a, b in zip(want, qs):
        assert_same_bytes(gpu_buffers(b), gpu_buffers(a))


def test_subnormal_bfloat16(q2d):
    """bfloat16 sums, outputs and gradients below the normal numbers keep their digits."""
    X = torch.full((3, 64), 2.0 ** -130, dtype=BF16, device=DEV)
    R = torch.full((3, 64), 2.0 ** -131, dtype=BF16, device=DEV)
    y, h, rstd = q2d.q2d_rmsnorm_fwd(X, torch.ones(64, device=DEV), 1.0, residual=R)
    assert bool((h.cpu().double() == 1.5 * 2.0 ** -130).all()) and bool((y.cpu().double() == 1.5 * 2.0 ** -130).all())
    dx, _ = q2d.q2d_rmsnorm_bwd(y, h, torch.ones(64, device=DEV), rstd, dh=h)
    assert bool((dx.cpu().double() == 3 * 2.0 ** -130).all())


def test_operands_in_place(q2d):
    for rows in (2, 40, 300):
        X, R, W = make((rows, 640), BF16, 27), make((rows, 640), BF16, 28), weight(640, F32)
        want, h, rstd = q2d.q2d_rmsnorm_quantize(X, W, residual=R, formats=(0, 1))
        for place in (0, 1):
            t = [X.clone(), R.clone()]
            got, h2, rstd2 = q2d.q2d_rmsnorm_quantize(t[0], W, residual=t[1], formats=(0, 1), h=t[place])
            assert torch.equal(h, h2) and torch.equal(rstd, rstd2)
            for a, b in zip(want, got):
                assert_same_bytes(gpu_buffers(b), gpu_buffers(a))


# ---------------------------------------------------------------- gradient

def gradient_case(shape, x, y, seed, scale=1e-3):
    X, W = make(shape, x, seed), None
    return X, (make(shape, F32, seed + 1) * scale).to(y), (make(shape, F32, seed + 2) * scale).to(x)


def check_backward(dx, dw, dy, h, W, rstd, dh):
    want, tol, want_w, tol_w = ref.backward(dy, h, W, rstd, dh)
    if dx.dtype == BF16:
        tol = tol + want.abs() * ref.unit(BF16) * (1 + 1e-3)
    assert bool(((dx.cpu().double() - want).abs() <= tol + 1e-44).all()), float(((dx.cpu().double() - want).abs() / tol).max())
    if dw is not None:
        assert bool(((dw.cpu().double() - want_w).abs() <= tol_w + 1e-44).all()), float(((dw.cpu().double() - want_w).abs() / tol_w).max())


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("x,y,w", [(BF16, BF16, F32), (F32, BF16, F32), (F32, F32, BF16), (BF16, F32, BF16)], ids=str)
def test_backward(q2d, shape, x, y, w):
    W = weight(shape[1], w)
    X, dy, dh = gradient_case(shape, x, y, 31)
    rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
    for d in (dh, None):
        check_backward(*q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=d), dy, X, W, rstd, d)


@pytest.mark.parametrize("cols,pad,shift", [(1000, 3, 1), (4096, 8, 0), (2049, 0, 0), (17000, 5, 2)])
def test_backward_rows_anywhere(q2d, cols, pad, shift):
    shape, W = (37, cols), weight(cols, F32)
    for x, y in ((BF16, F32), (F32, BF16)):
        X, dy, dh, dx = (make(shape, t, 40 + i, pad, shift) for i, t in enumerate((x, y, x, x)))
        rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
        got = q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh, dx=dx)
        check_backward(*got, dy, X, W, rstd, dh)
        if pad:
            assert bool((torch.as_strided(dx, (36, pad), (cols + pad, 1), dx.storage_offset() + cols) == 7).all())


@pytest.mark.parametrize("shape", [(700, 8200), (205, 8193), (1030, 16385), (1100, 5001), (515, 6144), (300, 12289)], ids=str)
@pytest.mark.parametrize("x,y", [(BF16, F32), (F32, BF16)], ids=str)
def test_backward_many_long_rows(q2d, shape, x, y):
    """More long rows than workgroups take in one turn, and a last turn that is short."""
    W = weight(shape[1], F32)
    X, dy, dh = gradient_case(shape, x, y, 45)
    rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
    check_backward(*q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh), dy, X, W, rstd, dh)


def test_backward_in_place_and_without_dw(q2d):
    for shape in ((70, 4096), (5, 20000), (400, 100)):
        W = weight(shape[1], F32)
        X, dy, dh = gradient_case(shape, BF16, BF16, 51)
        rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
        dx, dw = q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh)
        for place in ("dh", "dy"):
            t = {"dh": dh.clone(), "dy": dy.clone()}
            got = q2d.q2d_rmsnorm_bwd(t["dy"], X, W, rstd, dh=t["dh"], dx=t[place])
            assert got[0] is t[place] and torch.equal(got[0], dx) and torch.equal(got[1], dw)
        only, none = q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh, need_dw=False)
        assert none is None and torch.equal(only, dx)


def test_backward_against_differences(q2d):
    """The gradient of sum(y * dy) + sum(h * dh) by differences of the 64-bit form."""
    shape = (6, 40)
    W = weight(40, F32)
    X, dy, dh = gradient_case(shape, F32, F32, 61, 1.0)
    rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
    dx, dw = q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh)

    def f(x, w):
        return (ref.forward(x, w, EPS)[1] * dy.cpu().double()).sum() + (x * dh.cpu().double()).sum()

    x, w, step = X.cpu().double(), W.cpu().double(), 1e-5
    for t, got in ((x, dx), (w, dw)):
        for i in range(0, t.numel(), 7):
            d = torch.zeros_like(t)
            d.view(-1)[i] = step
            a = (x + d, w) if t is x else (x, w + d)
            b = (x - d, w) if t is x else (x, w - d)
            want = float(f(*a) - f(*b)) / (2 * step)
            # (the difference's error: its third derivative's step^2, and 64-bit cancellation)
            assert abs(float(got.view(-1)[i]) - want) <= 1e-4 * (1 + abs(want))


def test_many_rows(q2d):
    """Weights' gradients over many rows: sums in 64 bits."""
    for shape, x in (((100000, 96), BF16), ((40000, 520), F32)):
        W = weight(shape[1], F32)
        X, dy, dh = gradient_case(shape, x, BF16, 71)
        dy += 0.01
        rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
        check_backward(*q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh), dy, X, W, rstd, dh)


def test_same_results_again(q2d):
    W = weight(4096, F32)
    X, dy, dh = gradient_case((3000, 4096), BF16, BF16, 81)
    rstd = q2d.q2d_rmsnorm_fwd(X, W)[2]
    first = q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh)
    for _ in range(3):
        again = q2d.q2d_rmsnorm_bwd(dy, X, W, rstd, dh=dh)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
