"""Outputs beside inputs in one tensor, and in the place of the query or its gradient: accepted,
with the results of separate tensors."""
import pytest
import torch

from test_gpu_attention import make, q2d  # noqa: F401  (q2d: the fixture)
from test_gpu_kv_cache import filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv,D", [(4, 2, 64), (64, 64, 128), (2, 1, 128)])
def test_slices_of_one_tensor(q2d, H, Hkv, D):
    """q, k, v, the output and all gradients as heads of one tensor, for one sequence and two."""
    for B in (1, 2):
        q, k, v, dout = make(B, 150, 150, H, Hkv, D, torch.bfloat16, seed=101)
        out, lse = q2d.q2d_attention_fwd(q, k, v)
        grads = q2d.q2d_attention_bwd(dout, q, k, v, out, lse)
        heads = (H, Hkv, Hkv, H, H, H, Hkv, Hkv)
        x = torch.zeros((B, 150, sum(heads), D), dtype=torch.bfloat16, device="cuda").split(heads, 2)
        for t, s in zip(x, (q, k, v, dout)):
            t.copy_(s)
        o2, lse2 = q2d.q2d_attention_fwd(*x[:3], out=x[4])
        assert torch.equal(o2, out) and torch.equal(lse2, lse)
        for a, b in zip(q2d.q2d_attention_bwd(x[3], *x[:3], x[4], lse2, dq=x[5], dk=x[6], dv=x[7]), grads):
            assert torch.equal(a, b)


@pytest.mark.parametrize("H,D", [(2, 64), (64, 128)])
def test_in_place_of_the_query(q2d, H, D):
    q, k, v, dout = make(2, 150, 150, H, H, D, torch.bfloat16, seed=102)
    out, lse = q2d.q2d_attention_fwd(q, k, v)
    grads = q2d.q2d_attention_bwd(dout, q, k, v, out, lse)
    for where in (0, 3):
        t = [x.clone() for x in (q, k, v, dout)]
        got = q2d.q2d_attention_bwd(t[3], *t[:3], out, lse, dq=t[where])
        assert got[0].data_ptr() == t[where].data_ptr() and all(torch.equal(a, b) for a, b in zip(got, grads))
    t = q.clone()
    assert torch.equal(q2d.q2d_attention_fwd(t, k, v, out=t)[0], out)


@pytest.mark.parametrize("take", [1, 40])
def test_cached_in_place_of_the_query(q2d, take):
    p = filled(q2d, [1500, 90], 2, 64, capacity=1536)
    q = torch.randn((2 * take, 8, 64), generator=torch.Generator().manual_seed(103)).to(torch.bfloat16).cuda()
    want = q2d.q2d_attention_cached(q, p.cache, p.table.cuda(), p.lens().cuda())
    assert torch.equal(q2d.q2d_attention_cached(q, p.cache, p.table.cuda(), p.lens().cuda(), out=q), want)
