"""A distance bias at positions that float32 does not hold (past 2^24): queries at the end of a
long sequence under a window, so that only its last keys count and the definition can be taken
over these alone."""
import pytest
import torch

import attention_ref as ref
from test_gpu_attention import U, limits, q2d  # noqa: F401  (q2d: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype", [(8, torch.bfloat16), (8, torch.float32), (72, torch.bfloat16)], ids=str)
def test_distances_past_2_24(q2d, D, dtype):
    Lq, Lk, W, tail = 200, 2 ** 24 + 301, 150, 512
    g = torch.Generator().manual_seed(41)
    q, dout = (torch.randn((1, Lq, 1, D), generator=g).to(dtype).cuda() for _ in range(2))
    ends = [torch.randn((1, tail, 1, D), generator=g).to(dtype) for _ in range(2)]
    k, v = (torch.zeros((1, Lk, 1, D), dtype=dtype, device="cuda") for _ in range(2))
    k[:, -tail:], v[:, -tail:] = ends[0].cuda(), ends[1].cuda()
    slopes = torch.tensor([0.25])
    mask = dict(window=W, slopes=slopes.cuda())
    out, lse = q2d.q2d_attention_fwd(q, k, v, **mask)
    dq, dk, dv = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, **mask)
    want = ref.attention(q, *ends, dout, window=W, slopes=slopes)
    bound = limits(q, *ends, dout, dict(window=W, slopes=slopes), dtype)
    assert float((lse.cpu().double() - want[1]).abs().max()) <= 2.0 ** -14
    assert not dk[:, :-tail].any() and not dv[:, :-tail].any()
    for got, w, lim in zip((out, dq, dk[:, -tail:], dv[:, -tail:]), (want[0],) + want[2:], bound):
        assert bool(((got.cpu().double() - w).abs() <= lim + 1e-30).all())
