"""Errors of bfloat16 results in norm, in units of what rounding the exact result once costs.

Independent roundings add in squares, each of them one unit r at most:
* out and dV: the weights (P) and the result: sqrt(2) = 1.41; 1.5 is allowed.
* dQ and dK: dS, the result, and delta from the rounded out.  delta's share is below one unit:
  it moves dS by P eps |dO||O| where dS itself is P |dO||v - O| in size.  sqrt(3) = 1.73; 1.75 is
  allowed.
A second rounding of the weights, or of a sum to bfloat16, passes these limits."""
import pytest
import torch

import attention_ref as ref
from kv_ref import Paged
from test_gpu_attention import make, q2d  # noqa: F401  (q2d: the fixture)
from test_gpu_kv_cache import tokens

pytestmark = pytest.mark.gpu


def units(got, want):
    """Norm of the error over that of the exact result rounded once."""
    once = want.to(torch.bfloat16).double() - want
    return float((got.cpu().double() - want).norm() / once.norm())


DOCUMENTS = torch.tensor([[i // 130 for i in range(600)]], dtype=torch.int32)
CASES = {"causal": {}, "full": dict(causal=False), "cap": dict(softcap=3.0), "documents": dict(documents=DOCUMENTS),
         "bias": dict(slopes=torch.tensor([0.3, 0.01] * 4))}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", sorted(CASES))
def test_whole_sequences(q2d, name, D):
    q, k, v, dout = make(1, 600, 600, 8, 4, D, torch.bfloat16, seed=61)
    mask = CASES[name]
    dev = {n: (t.cuda() if isinstance(t, torch.Tensor) else t) for n, t in mask.items()}
    out, lse = q2d.q2d_attention_fwd(q, k, v, **dev)
    grads = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, **dev)
    want = ref.attention(q, k, v, dout, **mask)
    got = dict(zip(("out", "dq", "dk", "dv"), (units(a, b) for a, b in zip((out,) + tuple(grads), (want[0],) + want[2:]))))
    print(name, D, {n: round(x, 3) for n, x in got.items()}, flush=True)
    assert got["out"] <= 1.5 and got["dv"] <= 1.5 and got["dq"] <= 1.75 and got["dk"] <= 1.75, got


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("take", [1, 300])
def test_over_the_cache(q2d, take, D):
    batch = 16 if take == 1 else 2
    p = Paged(q2d, batch, 2, D, 64, 704)
    p.append(*tokens(700 * batch, 2, D, seed=62), [700] * batch)
    q = torch.randn((take * batch, 8, D), generator=torch.Generator().manual_seed(63)).to(torch.bfloat16).cuda()
    out = q2d.q2d_attention_cached(q, p.cache, p.table.cuda(), p.lens().cuda())
    want = torch.cat([ref.attention(q[b * take:(b + 1) * take][None], *(x[None] for x in p.dense(b)))[0][0]
                      for b in range(batch)])
    got = units(out, want)
    print(take, D, round(got, 3), flush=True)
    assert got <= 1.5
