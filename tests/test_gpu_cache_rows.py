"""Rows that no token of a sequence stands behind are zeros: rows of no sequence (a padded batch),
and for reads also tokens on missing pages and rows before a sequence's first position."""
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,dim", [(1, 16), (3, 80), (2, 128)])
def test_read(q2d, heads, dim, dtype):
    p = filled(q2d, [200, 65, 3], heads, dim)
    table = p.table.clone()
    table[0, 1], table[1, 0] = -1, p.cache.pages          # tokens 64 .. 127 and 0 .. 63 are on no page
    off = torch.tensor([2, 152, 217, 227])                # of 3 tokens, 10 rows
    k, v = (torch.full((240, heads, dim), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    q2d.q2d_kv_read(p.cache, table.cuda(), p.lens().cuda(), 240, off.cuda(), k=k, v=v)
    for got, which in ((k, 0), (v, 1)):
        want = torch.zeros((240, heads, dim), dtype=torch.float64)
        for b, (lo, hi, n) in enumerate(((2, 152, 200), (152, 217, 65), (217, 227, 3))):
            x = p.dense(b)[which]
            m = min(hi - lo, n)
            want[hi - m:hi] = x[n - m:]
        want[2 + 14:2 + 78] = 0                           # positions 50 .. 199 in rows 2 .. 151
        want[152:152 + 64] = 0
        assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("name", sorted(OFFSETS))
def test_read_of_no_sequence(q2d, name):
    p = filled(q2d, [70, 65, 60], 2, 64)
    k, v = (torch.full((12, 2, 64), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    off = torch.tensor(OFFSETS[name])
    q2d.q2d_kv_read(p.cache, p.table.cuda(), p.lens().cuda(), 12, off.cuda(), k=k, v=v)
    lo, hi = int(off[0].clamp(0, 12)), int(off[-1].clamp(0, 12))
    for x in (k, v):
        assert not x[:lo].any() and not x[hi:].any() and bool(x[lo:hi].any(-1).all()) and torch.isfinite(x).all()


def test_read_without_offsets(q2d):
    """Equally many rows each, more than the sequences have tokens."""
    p = filled(q2d, [5, 1, 0], 2, 64)
    k, v = (torch.full((24, 2, 64), math.nan, dtype=torch.float32, device="cuda") for _ in range(2))
    q2d.q2d_kv_read(p.cache, p.table.cuda(), p.lens().cuda(), 24, k=k, v=v)
    for x, which in ((k, 0), (v, 1)):
        want = torch.zeros((24, 2, 64), dtype=torch.float64)
        want[3:8], want[15:16] = p.dense(0)[which], p.dense(1)[which]
        assert torch.equal(x.cpu().double(), want)


def test_padded_batch_in_a_graph(q2d):
    """One captured call for up to 12 new tokens of three sequences, replayed with other counts: rows
    behind the last one are zeros each time, whatever the replay before left in them."""
    p = filled(q2d, [300, 65, 90], 2, 64)
    table, lens = p.table.cuda(), p.lens().cuda()
    q = torch.randn((12, 8, 64), generator=torch.Generator().manual_seed(72)).to(torch.bfloat16).cuda()
    off = torch.tensor([0, 4, 8, 12]).cuda()
    out, k, v = torch.empty_like(q), *(torch.empty((12, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step():
        q2d.q2d_attention_cached(q, p.cache, table, lens, off, out=out)
        q2d.q2d_kv_read(p.cache, table, lens, 12, off, k=k, v=v)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()                                  # the workspace's allocation, outside the capture
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for counts in ([4, 4, 4], [1, 0, 2], [3, 3, 0], [0, 0, 0], [12, 0, 0], [1, 1, 1]):
        ends = torch.tensor(counts).cumsum(0)
        off[1:].copy_(ends)
        graph.replay()
        torch.cuda.synchronize()
        n = int(ends[-1])
        got = [t.clone() for t in (out, k, v)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, k, v)):
            assert torch.equal(a, b) and not a[n:].any() and bool(a[:n].any(-1).all())
