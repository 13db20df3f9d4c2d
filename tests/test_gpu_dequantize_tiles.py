"""q2d_dequantize at sizes whose matrices are cut into whole tiles (more than 128 of 128 x 256), against the
oracle: all formats, both copies, ragged edges, exponents, outputs of any pitch and alignment, and the
bfloat16 outputs of 96 MB and more that are written past the cache."""
import pytest
import torch

import oracle
import synth
from test_gpu_dequantize import DEV, FMTS, check_copy, q2d, quantize_both      # noqa: F401

pytestmark = pytest.mark.gpu

# the last tile's rows and columns: 52 and 132, 1 and 77, 33 and 128; odd row pitches of the exponents
SHAPES = [(2100, 2180), (4225, 1101), (16417, 128)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("fmt", FMTS)
def test_tiles(q2d, shape, fmt):
    x = synth.normal(shape, 1.0, 910 + shape[0], torch.bfloat16, device=DEV)
    synth.add_outlier_channels(x, 9, frac=0.03)
    x[3, 40], x[shape[0] - 1, shape[1] - 1], x[700, 100] = float("nan"), float("inf"), 3e38
    q, o = quantize_both(q2d, x, fmt)
    for copy in (0, 1):
        for dt in (torch.float32, torch.bfloat16):
            print(shape, fmt, copy, dt, flush=True)
            check_copy(q2d, q, o, fmt, copy, dt, "%s %s copy %d %s" % (shape, fmt, copy, dt))
            big = torch.full((shape[0], shape[1] + 11), 7.0, dtype=dt, device=DEV)
            check_copy(q2d, q, o, fmt, copy, dt, "strided", out=big[:, 1:1 + shape[1]])
            assert bool((big[:, 0] == 7).all()) and bool((big[:, 1 + shape[1]:] == 7).all())


@pytest.mark.parametrize("shape", [(2100, 2180), (130, 200), (33, 129), (5, 3)], ids=str)
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_exponents_anywhere(q2d, shape, fmt, pad, shift):
    """Exponents of any pitch and alignment; what lies between their rows is left alone."""
    rows, cols = shape
    x = synth.normal(shape, 1.0, 911, torch.bfloat16, device=DEV)
    x[rows - 1, 0] = float("nan")
    q, o = quantize_both(q2d, x, fmt)
    out = torch.empty(shape, device=DEV)
    for copy in (0, 1):
        buf = torch.full((rows * (cols + pad) + shift,), 77, dtype=torch.int8, device=DEV)
        e = torch.as_strided(buf, shape, (cols + pad, 1), shift)
        assert q2d._lib.q2d_dequantize(q.ptr(), copy, out.data_ptr(), 0, cols, e.data_ptr(), cols + pad,
                                       torch.cuda.current_stream().cuda_stream) == 0
        want = torch.from_numpy(oracle.scale_exponents(o, copy, "fp4" if fmt == "fp4_b64" else fmt)).to(torch.int8)
        assert torch.equal(e.cpu(), want) and int(e[rows - 1, 0]) == -128
        assert bool((buf[:shift] == 77).all())
        if pad:
            assert bool((torch.as_strided(buf, (rows, pad), (cols + pad, 1), shift + cols) == 77).all())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", [(8200, 6150), (16384, 4096)], ids=str)
def test_output_past_the_cache(q2d, fmt, shape):
    """bfloat16 output of 96 MB and more is the rounded float32 output."""
    x = synth.normal(shape, 1.0, 912, torch.bfloat16, device=DEV)
    synth.add_outlier_channels(x, 10, frac=0.03)
    x[5, 5], x[100, shape[1] - 1], x[shape[0] - 1, 64] = float("nan"), float("inf"), 3.3e38
    q = (q2d.mxfp8_quantize(x) if fmt == "mxfp8" else q2d.q2d_quantize_1d(x) if fmt == "fp4_1d" else
         q2d.q2d_quantize(x, block=64 if fmt == "fp4_b64" else 32))
    for copy in (0, 1):
        want, e = q2d.q2d_dequantize(q, copy, exps=True)
        big = torch.full((shape[0], shape[1] + 3), 7.0, dtype=torch.bfloat16, device=DEV)
        for out in (None, big[:, 1:1 + shape[1]]):
            print(shape, fmt, copy, out is None, flush=True)
            got, e2 = q2d.q2d_dequantize(q, copy, torch.bfloat16, exps=True, out=out)
            assert torch.equal(e, e2) and torch.equal(got.isnan(), want.isnan())
            assert torch.equal(got.nan_to_num(0.0), want.to(torch.bfloat16).nan_to_num(0.0))
        assert bool((big[:, 0] == 7).all()) and bool((big[:, 1 + shape[1]:] == 7).all())


# strips, tiles, and bfloat16 past the cache
@pytest.mark.parametrize("repeat", [(1, 1), (9, 20), (33, 25)], ids=str)
@pytest.mark.parametrize("fmt", ["fp4_1d", "mxfp8"])
@pytest.mark.parametrize("copy", [0, 1])
def test_every_code_and_scale(q2d, fmt, copy, repeat):
    """All codes under all scale bytes, one scale byte a line; every NaN is 0x7FC00000 (0x7FC0)."""
    lines, width = 256 * repeat[0], 256 * repeat[1]
    shape = (lines, width) if copy == 0 else (width, lines)
    q = q2d.QTensor(q2d.MXFP8 if fmt == "mxfp8" else q2d.FP4_1D, *shape, DEV, 32, (copy == 0, copy == 1))
    codes, scales = (q.codes, q.scales) if copy == 0 else (q.codes_t, q.scales_t)
    byte = torch.arange(256).repeat(repeat[0]).to(torch.uint8)
    if fmt == "mxfp8":
        one = torch.arange(256).repeat(repeat[1]).to(torch.uint8)
        values = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).repeat(repeat[1])
        scales.copy_(byte[:, None].expand(scales.shape))
    else:
        nibbles = torch.arange(256).repeat(repeat[1]) % 16
        one = (nibbles[::2] | nibbles[1::2] << 4).to(torch.uint8)
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
        values = torch.cat((table, -table))[nibbles]
        scales.copy_(byte.repeat_interleave(4)[None].expand(scales.shape))
    codes.copy_(one[None].expand(codes.shape))
    want = torch.ldexp(values[None], byte[:, None].to(torch.int64) - 127)
    want[byte == 255] = float("nan")
    want = want.float() if copy == 0 else want.float().t()
    bad = want.isnan()
    for dt, bits in ((torch.float32, torch.int32), (torch.bfloat16, torch.int16)):
        print(fmt, copy, repeat, dt, flush=True)
        got = q2d.q2d_dequantize(q, copy, dt).cpu()
        w = want.to(dt).contiguous().view(bits)
        w[bad] = 0x7FC00000 if dt == torch.float32 else 0x7FC0
        assert torch.equal(got.view(bits), w)
