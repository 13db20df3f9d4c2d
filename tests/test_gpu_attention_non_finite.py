"""Infinities and NaN that are seen: results as the definition has them, in tiles with masked pairs
and without, at ragged ends.  Compared is which elements are finite; where only an infinity can
come out, that it does."""
import math

import pytest
import torch

from test_gpu_attention import make, q2d  # noqa: F401  (q2d: the fixture)

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
DIMS = pytest.mark.parametrize("D", [64, 96, 128])


@DTYPES
@pytest.mark.parametrize("H", [1, 260])
@DIMS
@pytest.mark.parametrize("Lq,causal", [(100, False), (1, True), (33, False)], ids=str)
def test_infinite_last_value(q2d, Lq, causal, D, H, dtype):
    """The last key of a ragged tile, which every query sees."""
    q, k, v, _ = make(1, Lq, 100, H, H, D, dtype, seed=51)
    base = q2d.q2d_attention_fwd(q, k, v, causal=causal)[0]
    v[:, 99, :, 3] = math.inf
    out = q2d.q2d_attention_fwd(q, k, v, causal=causal)[0]
    assert bool((out[..., 3] == math.inf).all())
    rest = [d for d in range(D) if d != 3]
    assert torch.equal(out[..., rest], base[..., rest])
