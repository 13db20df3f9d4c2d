"""Matrices whose tiles pass what one dimension of a launch takes: 2^30 rows and more of one column."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
ROWS = (1 << 30) + 300
STEP = 1 << 28                          # rows that one dimension takes


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def fill(t, seed):
    """Random bytes in place, a piece at a time."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    for p in t.view(-1).split(1 << 26):
        p.copy_(torch.randint(256, (p.numel(),), dtype=torch.uint8, generator=g, device=DEV))


def piece(q2d, q, first):
    """Up to STEP rows of a column's transposed copy, from row `first` on, as a matrix of their own."""
    t = q2d.QTensor(q.fmt, min(STEP, q.rows - first), 1, DEV, 32, (False, True))
    at = first if q.fmt == q2d.MXFP8 else first // 2
    t.codes_t.copy_(q.codes_t[:, at:at + t.codes_t.shape[1]])
    if q.fmt == q2d.FP4_1D:
        t.scales_t.copy_(q.scales_t[first // 128:first // 128 + t.scales_t.shape[0]])
    else:
        t.scales_t.copy_(q.scales_t[:, first // 32:first // 32 + t.scales_t.shape[1]])
    return t


@pytest.mark.parametrize("fmt", ["FP4_2D", "FP4_1D", "MXFP8"])
def test_dequantize_column(q2d, fmt):
    q = q2d.QTensor(getattr(q2d, fmt), ROWS, 1, DEV, 32, (False, True))
    fill(q.codes_t, 1)
    fill(q.scales_t, 2)
    out = torch.full((ROWS, 1), 7.0, dtype=torch.bfloat16, device=DEV)
    print("dequantize", fmt, ROWS, flush=True)
    q2d.q2d_dequantize(q, 1, out=out)
    for first in range(0, ROWS, STEP):
        want = q2d.q2d_dequantize(piece(q2d, q, first), 1, torch.bfloat16)
        got = out[first:first + STEP]
        assert torch.equal(got.isnan(), want.isnan()), first
        assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0)), first


@pytest.mark.parametrize("fmt", ["FP4_1D", "MXFP8"])
def test_norm_operand_column(q2d, fmt):
    x = torch.empty((ROWS, 1), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    for p in x.view(-1).split(1 << 26):
        p.copy_(1e-2 * torch.randn(p.numel(), generator=g, device=DEV))
    w, f = torch.tensor([1.3], device=DEV), getattr(q2d, fmt)
    print("norm operand", fmt, ROWS, flush=True)
    (q,), _, rstd = q2d.q2d_rmsnorm_quantize(x, w, 1e-4, formats=(f,), orientations=(False, True))
    for first in range(0, ROWS, STEP):
        rows = x[first:first + STEP]
        (want,), _, rs = q2d.q2d_rmsnorm_quantize(rows, w, 1e-4, formats=(f,), orientations=(False, True))
        got = piece(q2d, q, first)
        assert torch.equal(rstd[first:first + STEP], rs) and torch.equal(got.codes_t, want.codes_t), first
        assert torch.equal(got.scales_t, want.scales_t), first
        # (and the first and last of them by the separate quantizer)
        for a in (0, rows.shape[0] - 128 - rows.shape[0] % 128):
            y = q2d.q2d_rmsnorm_fwd(rows[a:a + 128], w, 1e-4, y_dtype=torch.float32)[0]
            own = q2d.mxfp8_quantize(y) if fmt == "MXFP8" else q2d.q2d_quantize_1d(y)
            at = a if fmt == "MXFP8" else a // 2
            assert torch.equal(got.codes_t[:, at:at + own.codes_t.shape[1]], own.codes_t), (first, a)
