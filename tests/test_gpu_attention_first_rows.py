"""dQ and dK where rows see few keys: the beginnings of sequences and of many short documents.

delta = rowsum(dO * O) of an O rounded to bfloat16 is off by one rounding's unit r of |dO||O|, which
moves a row's dS by P of it: beside r times the row's own dS only while it sees few keys (1 / n of
its square), but there the most, and for a row that sees one key, whose dS is 0, all there is.
With delta exact for these rows, dS and the result are rounded once each: sqrt(2) = 1.41 units of
rounding the exact result once, and what delta adds for rows of more than 8 keys is below a
tenth in squares: 1.5 is allowed, as for out and dV."""
import pytest
import torch

import attention_ref as ref
from test_gpu_attention import make, q2d  # noqa: F401  (q2d: the fixture)
from test_gpu_attention_accuracy import units

pytestmark = pytest.mark.gpu


def documents(sizes, L):
    d, at = torch.full((1, L), -1, dtype=torch.int32), 0
    i = 0
    while at < L:
        n = sizes[i % len(sizes)]
        d[0, at:at + n] = i
        at, i = at + n, i + 1
    return d


CASES = {"short documents": dict(documents=documents([5, 12, 1, 20, 33, 2, 9], 600)),
         "documents": dict(documents=documents([130, 77], 600)),
         "mixed documents": dict(documents=torch.tensor([[i % 37 for i in range(600)]], dtype=torch.int32)),
         "narrow window": dict(window=6), "cap": dict(softcap=3.0, documents=documents([9, 31], 600)),
         "bias": dict(slopes=torch.tensor([0.3, 0.01] * 4), documents=documents([40], 600)), "causal": {}}


# Few keys, but not among the row's own position and the seven before it: delta stays that of the
# rounded O, and the errors within the 1.75 units of the other accuracy tests.
NOT_REACHED = pytest.mark.xfail(strict=True, reason="rows whose few keys lie apart, or fade out over tens of positions")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", [pytest.param(n, marks=NOT_REACHED) if n in ("bias", "mixed documents") else n
                                  for n in sorted(CASES)])
def test_gradients(q2d, name, D):
    q, k, v, dout = make(1, 600, 600, 8, 4, D, torch.bfloat16, seed=111)
    mask = CASES[name]
    dev = {n: (t.cuda() if isinstance(t, torch.Tensor) else t) for n, t in mask.items()}
    out, lse = q2d.q2d_attention_fwd(q, k, v, **dev)
    grads = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, **dev)
    want = ref.attention(q, k, v, dout, **mask)[2:]
    got = {n: units(a, b) for n, a, b in zip(("dq", "dk", "dv"), grads, want)}
    print(name, D, {n: round(x, 3) for n, x in got.items()}, flush=True)
    assert max(got.values()) <= 1.5, got


def test_one_key_a_row(q2d):
    """Rows that see themselves alone: their scores have no gradient."""
    q, k, v, dout = make(1, 300, 300, 4, 2, 64, torch.bfloat16, seed=112)
    out, lse = q2d.q2d_attention_fwd(q, k, v, window=1)
    dq, dk, _ = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, window=1)
    # float32's rounding of sums of 64 products, of size 8, times scale and |k| or |q|
    size = 2.0 ** -20 * 8 * 64 ** -0.5
    assert float(dq.abs().max()) <= size * float(k.abs().max()) and float(dk.abs().max()) <= 2 * size * float(q.abs().max())
