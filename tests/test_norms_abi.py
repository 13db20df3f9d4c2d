"""Host-side checks of the norm's and the gradients' entry points (no GPU, no kernel is launched)."""
import ctypes

import pytest
import torch

FAKE = 0x100000
MB = 1 << 20


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def norm(q2d, **kw):
    from paper_2607_24953_amd import norms as N
    n = N._Norm(x_dtype=1, residual_dtype=1, weight_dtype=0, y_dtype=1, rows=16, cols=64, eps=1e-5, x=FAKE, ldx=64,
                residual=FAKE + MB, ld_residual=64, weight=FAKE + 2 * MB, h=FAKE + 3 * MB, ldh=64, y=FAKE + 4 * MB, ldy=64,
                rstd=FAKE + 5 * MB)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def tensor(q2d, fmt, rows=16, cols=64, at=FAKE + 6 * MB, **kw):
    t = q2d._Tensor()
    assert q2d._lib.q2d_tensor_init(ctypes.byref(t), fmt, rows, cols, 32, None) == 0
    for i, name in enumerate(("codes", "codes_t", "scales", "scales_t")):
        setattr(t, name, at + i * MB)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def fwd(q2d, n, q4=None, q8=None):
    ref = lambda t: None if t is None else ctypes.byref(t)
    return q2d._lib.q2d_rmsnorm_fwd(ref(n), ref(q4), ref(q8), None)


@pytest.mark.parametrize("bad,status", [
    (dict(x_dtype=2), 1), (dict(residual_dtype=-1), 1), (dict(weight_dtype=7), 1), (dict(y_dtype=2), 1), (dict(rows=-1), 1),
    (dict(cols=0), 1), (dict(cols=-5), 1), (dict(rows=2 ** 31 + 1), 2), (dict(rows=2 ** 31), 2), (dict(cols=2 ** 27 + 1, ldx=2 ** 28), 2), (dict(eps=0.0), 1),
    (dict(eps=-1e-5), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(eps=1e-39), 1), (dict(x=None), 1),
    (dict(weight=None), 1), (dict(rstd=None), 1), (dict(rstd=FAKE + 5 * MB + 2), 1), (dict(h=None), 1), (dict(residual=None), 1),
    (dict(y=None), 1), (dict(ldx=63), 1), (dict(ldh=0), 1), (dict(ldy=-64), 1), (dict(ld_residual=32), 1), (dict(x=FAKE + 1), 1),
    (dict(weight=FAKE + 2 * MB + 2), 1), (dict(ldx=2 ** 44), 2), (dict(ldx=2 ** 62), 2), (dict(rows=2 ** 20, ldy=2 ** 28), 2),
    # memory that is still read or written elsewhere
    (dict(y=FAKE), 1), (dict(y=FAKE + MB), 1), (dict(y=FAKE + 3 * MB), 1), (dict(h=FAKE + 2), 1), (dict(h=FAKE + 64), 1),
    (dict(h=FAKE, ldh=65), 1), (dict(y=FAKE + 2 * MB), 1), (dict(rstd=FAKE), 1), (dict(rstd=FAKE + 4 * MB), 1),
    (dict(residual_dtype=0, h=FAKE + MB), 1), (dict(y=FAKE + 32 * 2, ldx=100, ldy=100), 1), (dict(rstd=FAKE + 2 * MB), 1),
], ids=str)
def test_forward_refusals(q2d, bad, status):
    assert fwd(q2d, norm(q2d, **bad)) == status


def test_forward_operand_refusals(q2d):
    assert fwd(q2d, None) == 1
    one = dict(y=None)
    F = lambda q4=None, q8=None, **kw: fwd(q2d, norm(q2d, **{**one, **kw}), q4, q8)
    assert F(tensor(q2d, q2d.MXFP8)) == 1 and F(None, tensor(q2d, q2d.FP4_2D)) == 1 and F(None, tensor(q2d, q2d.FP4_1D)) == 1
    assert F(tensor(q2d, q2d.FP4_2D, rows=17)) == 1 and F(None, tensor(q2d, q2d.MXFP8, cols=65)) == 1
    assert F(tensor(q2d, q2d.FP4_2D), rows=0) == 1
    assert F(tensor(q2d, q2d.FP4_2D, codes=None, codes_t=None)) == 1 and F(tensor(q2d, q2d.FP4_2D, scales=None)) == 1
    assert F(tensor(q2d, q2d.FP4_2D, codes=FAKE + 6 * MB + 8)) == 1 and F(tensor(q2d, q2d.FP4_2D, ld_codes=16)) == 1
    assert F(tensor(q2d, q2d.FP4_2D, block=16)) == 2 and F(tensor(q2d, q2d.FP4_1D, block=64)) == 2
    # operands in one another's memory, or in that of what is read
    assert F(tensor(q2d, q2d.FP4_2D), tensor(q2d, q2d.MXFP8)) == 1
    assert F(tensor(q2d, q2d.FP4_2D, codes=FAKE)) == 1 and F(None, tensor(q2d, q2d.MXFP8, codes_t=FAKE + 3 * MB)) == 1
    assert F(tensor(q2d, q2d.FP4_2D, scales=FAKE + 2 * MB)) == 1 and F(tensor(q2d, q2d.FP4_1D, scales_t=FAKE + 5 * MB)) == 1


def test_no_rows(q2d):
    assert fwd(q2d, norm(q2d, rows=0)) == 0


def grad(q2d, **kw):
    from paper_2607_24953_amd import norms as N
    n = N._NormGrad(h_dtype=1, dy_dtype=1, weight_dtype=0, rows=16, cols=64, h=FAKE, ldh=64, dy=FAKE + MB, lddy=64,
                    dh=FAKE + 2 * MB, lddh=64, dx=FAKE + 3 * MB, lddx=64, weight=FAKE + 4 * MB, rstd=FAKE + 5 * MB,
                    dw=FAKE + 6 * MB)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


@pytest.mark.parametrize("bad,status", [
    (dict(h_dtype=2), 1), (dict(dy_dtype=2), 1), (dict(weight_dtype=2), 1), (dict(rows=-1), 1), (dict(cols=0), 1),
    (dict(rows=2 ** 31), 2), (dict(cols=2 ** 27 + 1), 2), (dict(h=None), 1), (dict(dy=None), 1), (dict(dx=None), 1), (dict(weight=None), 1),
    (dict(rstd=None), 1), (dict(ldh=1), 1), (dict(lddx=63), 1), (dict(dw=FAKE + 6 * MB + 2), 1), (dict(lddy=2 ** 60), 2),
    (dict(dx=FAKE), 1), (dict(dx=FAKE + MB, dy_dtype=0), 1), (dict(dx=FAKE + MB + 2), 1), (dict(dx=FAKE + 2 * MB, lddx=65), 1),
    (dict(dx=FAKE + 4 * MB), 1), (dict(dw=FAKE), 1), (dict(dw=FAKE + 3 * MB), 1), (dict(dw=FAKE + 5 * MB), 1),
    (dict(dx=FAKE + 16 * MB), 1), (dict(dw=FAKE + 16 * MB), 1), (dict(dy=FAKE + 16 * MB), 1),
], ids=str)
def test_backward_refusals(q2d, bad, status):
    n = grad(q2d, **bad)
    size = max(0, q2d._lib.q2d_rmsnorm_workspace(n.rows, n.cols))
    assert q2d._lib.q2d_rmsnorm_bwd(ctypes.byref(n), FAKE + 16 * MB, size, None) == status


def test_backward_workspace(q2d):
    W = q2d._lib.q2d_rmsnorm_workspace
    assert W(-1, 64) == -1 and W(16, 0) == -1 and W(2 ** 31 + 1, 64) == -1
    size = W(16, 64)
    assert size > 0
    B = lambda ws, n: q2d._lib.q2d_rmsnorm_bwd(ctypes.byref(grad(q2d)), ws, n, None)
    assert B(None, size) == 1 and B(FAKE + 16 * MB, size - 1) == 1 and B(FAKE + 16 * MB + 64, size) == 1
    assert q2d._lib.q2d_rmsnorm_bwd(None, FAKE, size, None) == 1


def clip(q2d, data, out=None, counts=None, dtypes=None, max_norm=1.0, given=None, norm=FAKE + 32 * MB, ws=FAKE + 33 * MB, size=None):
    n = len(data)
    arr = lambda t, v: None if v is None else (t * n)(*v)
    size = q2d._lib.q2d_grad_workspace(n) if size is None else size
    return q2d._lib.q2d_clip_grads(n, arr(ctypes.c_void_p, data), arr(ctypes.c_void_p, out),
                                   arr(ctypes.c_int64, counts if counts is not None else [64] * n),
                                   arr(ctypes.c_int32, dtypes if dtypes is not None else [0] * n), max_norm, given, norm, ws, size, None)


def test_clip_refusals(q2d):
    a, b, c, d = (FAKE + i * MB for i in range(4))
    for kw in (dict(dtypes=[0, 2]), dict(counts=[64, -1]), dict(max_norm=-1.0), dict(max_norm=float("nan")),
               dict(max_norm=float("inf")), dict(norm=None), dict(given=d, norm=c), dict(given=d + 1, norm=None), dict(ws=None),
               dict(ws=FAKE + 33 * MB + 4), dict(size=8), dict(out=[c, None]), dict(out=[c, c]), dict(out=[c, c + 128]),
               dict(out=[b, a]), dict(out=[a + 4, b]), dict(out=[c, d + 2]), dict(norm=FAKE + 32 * MB + 2),
               dict(norm=a), dict(norm=b + 252), dict(ws=a), dict(ws=b - 64), dict(out=[c, d], norm=a + 8), dict(given=b + 4, norm=None),
               dict(norm=FAKE + 33 * MB + 8)):
        assert clip(q2d, [a, b], **kw) == 1, kw
    assert clip(q2d, [a, None]) == 1 and clip(q2d, [a, a]) == 1 and clip(q2d, [a, a + 64]) == 1 and clip(q2d, [a, b + 1]) == 1
    assert clip(q2d, [a], counts=[2 ** 40 + 1]) == 2
    assert q2d._lib.q2d_clip_grads(-1, None, None, None, None, 1.0, None, FAKE, FAKE, 1 << 20, None) == 1
    assert q2d._lib.q2d_clip_grads(1, None, None, None, None, 1.0, None, FAKE, FAKE, 1 << 20, None) == 1
    assert q2d._lib.q2d_grad_workspace(-1) == -1 and q2d._lib.q2d_grad_workspace(0) > 0
    N = q2d._lib.q2d_grad_norm
    one = ((ctypes.c_void_p * 1)(a), (ctypes.c_int64 * 1)(5), (ctypes.c_int32 * 1)(0))
    size = q2d._lib.q2d_grad_workspace(1)
    assert N(1, *one, None, b, size, None) == 1 and N(1, *one, c, None, size, None) == 1 and N(1, *one, c, b, size - 1, None) == 1
    assert N(1, *one, c + 1, b, size, None) == 1 and N(1, one[0], one[1], (ctypes.c_int32 * 1)(9), c, b, size, None) == 1


def test_gradients_norm_memory(q2d):
    """The norm's place and the workspace, which are written while the tensors are read."""
    size = q2d._lib.q2d_grad_workspace(2)
    arr = lambda t, v: (t * 2)(*v)

    def call(norm, ws, data=(FAKE, FAKE + MB), counts=(1024, 1000)):
        return q2d._lib.q2d_grad_norm(2, arr(ctypes.c_void_p, data), arr(ctypes.c_int64, counts), arr(ctypes.c_int32, (0, 1)), norm, ws,
                                      size, None)
    free = FAKE + 4 * MB
    for norm, ws in ((FAKE, free), (FAKE + 4092, free), (FAKE + MB + 1996, free), (free, free), (free + size - 4, free),
                     (free, FAKE + 4088), (free, FAKE - size + 8), (free, FAKE + MB + 1992), (free, FAKE + MB - 8)):
        assert call(norm, ws) == 1, (norm, ws)
    # tensors without elements have no memory; the next byte is another's
    assert call(free, free, counts=(0, 0)) == 1
    for norm, ws in ((free, FAKE + 4096), (FAKE + 4096, free), (free + size, free), (free, FAKE - size)):
        assert call(norm, ws) != 1, (norm, ws)


def test_python_refusals(q2d):
    """Host tensors and mismatched arguments never reach the library."""
    x, w = torch.zeros((4, 8)), torch.ones(8)
    for call in (lambda: q2d.q2d_rmsnorm_fwd(x, w), lambda: q2d.q2d_rmsnorm_quantize(x, w), lambda: q2d.q2d_rmsnorm_fwd(x[0], w),
                 lambda: q2d.q2d_rmsnorm_bwd(x, x, w, w[:4]), lambda: q2d.q2d_grad_norm([x]), lambda: q2d.q2d_clip_grads([x], 1.0),
                 lambda: q2d.q2d_grad_norm([]), lambda: q2d.q2d_grad_norm([None])):
        with pytest.raises(q2d.Q2DError):
            call()
