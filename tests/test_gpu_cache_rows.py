"""Rows of no sequence (a padded batch) are zeros."""
import math

import pytest
import torch

from test_gpu_kv_cache import filled, q2d  # noqa: F401  (q2d: the fixture)

pytestmark = pytest.mark.gpu

OFFSETS = {"ends": [3, 4, 4, 10], "none before": [0, 1, 2, 3], "no rows": [5, 5, 5, 5], "all": [0, 6, 7, 12],
           "past the tensor": [2, 5, 90, 100]}


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 32)], ids=["16 rows", "128 rows"])
@pytest.mark.parametrize("name", sorted(OFFSETS))
@pytest.mark.parametrize("length", [70, 1500])
def test_attention(q2d, length, name, heads, group, dim):
    """(1500 tokens of one head: the sequences are cut into parts)"""
    p = filled(q2d, [length, 65, length - 10], heads, dim, capacity=1536)
    n = 12 if name != "none before" else 40
    q = torch.randn((n, heads * group, dim), generator=torch.Generator().manual_seed(71)).to(torch.bfloat16).cuda()
    off = torch.tensor(OFFSETS[name])
    args = (p.cache, p.table.cuda(), p.lens().cuda(), off.cuda())
    # a strided output, what it held before is anything
    out = torch.full((n, heads * group, 2 * dim), math.nan, dtype=torch.bfloat16, device="cuda")[..., :dim]
    q2d.q2d_attention_cached(q, *args, out=out)
    lo, hi = int(off[0].clamp(0, n)), int(off[-1].clamp(0, n))
    assert not out[:lo].any() and not out[hi:].any()
    assert torch.isfinite(out).all() and bool(out[lo:hi].any(-1).all())
    # the rows between are those of a call without the others
    if lo < hi:
        off = (off.clamp(0, n) - lo).cuda()
        assert torch.equal(q2d.q2d_attention_cached(q[lo:hi].contiguous(), *args[:3], off), out[lo:hi])


def test_attention_leaves_the_gaps_of_a_strided_output(q2d):
    p = filled(q2d, [70], 1, 64)
    out = torch.full((9, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    q2d.q2d_attention_cached(torch.ones((9, 4, 64), dtype=torch.bfloat16, device="cuda"), p.cache, p.table.cuda(),
                             p.lens().cuda(), torch.tensor([1, 3]).cuda(), out=out[..., :64])
    assert bool((out[..., 64:] == 7).all()) and not out[3:, :, :64].any() and not out[:1, :, :64].any()
