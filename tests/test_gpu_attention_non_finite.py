"""Infinities and NaN that are seen: results as the definition has them, in tiles with masked pairs
and without, at ragged ends.  Compared is which elements are finite; where only an infinity can
come out, that it does."""
import math

import pytest
import torch

import attention_ref as ref
from test_gpu_attention import make, q2d  # noqa: F401  (q2d: the fixture)

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
# few heads (32 rows a workgroup) and many (128 rows)
HEADS = pytest.mark.parametrize("H", [1, 130])
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


@DTYPES
@pytest.mark.parametrize("H", [1, 260])
@DIMS
def test_infinite_last_output_gradient(q2d, D, H, dtype):
    q, k, v, dout = make(1, 100, 100, H, H, D, dtype, seed=52)
    dout[:, 99, :, 3] = math.inf
    out, lse = q2d.q2d_attention_fwd(q, k, v, causal=False)
    dq, dk, dv = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, causal=False)
    assert bool((dv[..., 3] == math.inf).all())
    rest = [d for d in range(D) if d != 3]
    assert torch.isfinite(dv[..., rest]).all() and torch.isfinite(dq[:, :99]).all()
    assert not torch.isfinite(dk).any() and not torch.isfinite(dq[:, 99]).any()


def pattern(q2d, args, **mask):
    """Which elements are finite, against the definition, for out, dq, dk and dv."""
    q, k, v, dout = args
    dev = {n: (t.cuda() if isinstance(t, torch.Tensor) else t) for n, t in mask.items()}
    out, lse = q2d.q2d_attention_fwd(q, k, v, **dev)
    got = (out,) + tuple(q2d.q2d_attention_bwd(dout, q, k, v, out, lse, **dev))
    # (heads are alike: the first and the last stand for all)
    ends = sorted({0, q.shape[2] - 1})
    small = [t[:, :, ends] for t in args]
    want = ref.attention(*small, **mask)
    for name, a, b in zip(("out", "dq", "dk", "dv"), got, (want[0],) + want[2:]):
        assert torch.equal(torch.isfinite(a[:, :, ends]).cpu(), torch.isfinite(b)), name
    return got


DOCUMENTS = torch.tensor([[0] * 50 + [-1] * 9 + [1] * 101], dtype=torch.int32)
MASKS = {"causal": {}, "full": dict(causal=False), "window": dict(window=45), "documents": dict(documents=DOCUMENTS),
         "cap": dict(softcap=5.0), "cap window": dict(softcap=500.0, window=70)}


@DTYPES
@HEADS
@DIMS
@pytest.mark.parametrize("fill", [math.inf, math.nan])
@pytest.mark.parametrize("name", sorted(MASKS))
def test_output_gradient(q2d, name, fill, D, H, dtype):
    """One component of one dO row: only that component of dV is not finite."""
    args = make(1, 160, 160, H, H, D, dtype, seed=53)
    args[3][:, 90, :, 5] = fill
    dv = pattern(q2d, args, **MASKS[name])[3]
    assert torch.isfinite(dv[..., 6]).all() and not torch.isfinite(dv[:, 90, :, 5]).any()


@DTYPES
@HEADS
@DIMS
@pytest.mark.parametrize("fill", [math.inf, math.nan])
@pytest.mark.parametrize("name", sorted(MASKS))
def test_query(q2d, name, fill, D, H, dtype):
    """One component of one query.  Its scores are not finite; under a cap those of an infinity are,
    and only the component's own gradient with respect to the keys is not."""
    args = make(1, 160, 160, H, H, D, dtype, seed=54)
    args[0][:, 90, :, 5] = fill
    dk = pattern(q2d, args, **MASKS[name])[2]
    if "cap" in name and fill == math.inf:
        assert torch.isfinite(dk[..., 6]).all() and not torch.isfinite(dk[:, 90, :, 5]).any()


@DTYPES
@HEADS
@DIMS
@pytest.mark.parametrize("name", sorted(MASKS))
def test_key_with_scores_of_minus_infinity(q2d, name, D, H, dtype):
    """A key whose scores are all -infinity has weights of 0: only its own component of dQ (0 times
    an infinity) is not finite.  Under a cap its weights are those of -cap."""
    args = make(1, 160, 160, H, H, D, dtype, seed=55)
    args[0][..., 5] = -1.0 - args[0][..., 5].abs()
    args[1][:, 80, :, 5] = math.inf
    dq = pattern(q2d, args, **MASKS[name])[1]
    assert torch.isfinite(dq[..., 6]).all() and not torch.isfinite(dq[:, 80, :, 5]).any()


@DTYPES
@HEADS
@DIMS
@pytest.mark.parametrize("name", ["causal", "documents"])
def test_value(q2d, name, D, H, dtype):
    args = make(1, 160, 160, H, H, D, dtype, seed=56)
    args[2][:, 80, :, 5] = math.nan
    pattern(q2d, args, **MASKS[name])


@DTYPES
@pytest.mark.parametrize("D", [64, 128])
def test_shared_heads_in_parts(q2d, D, dtype):
    """The sums in parts: one query head's infinity reaches the shared head's gradients alike."""
    q, k, v, dout = make(1, 1100, 1100, 4, 1, D, dtype, seed=57)
    dout[:, 700, 2, 5] = math.inf
    out, lse = q2d.q2d_attention_fwd(q, k, v, window=300)
    dq, dk, dv = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, window=300)
    sees = torch.zeros(1100, dtype=torch.bool, device="cuda")
    sees[401:701] = True
    assert torch.equal(dv[0, :, 0, 5] == math.inf, sees)
    dv[..., 5] = 0
    assert torch.isfinite(dv).all()
    assert torch.equal(torch.isfinite(dk[0, :, 0]).all(-1), ~sees)
    assert torch.isfinite(dq[:, :, [0, 1, 3]]).all()


@DTYPES
@HEADS
@DIMS
@pytest.mark.parametrize("name", ["causal", "documents", "window"])
def test_rows_with_scores_of_minus_infinity_alone(q2d, name, D, H, dtype):
    """A softmax over nothing but -infinity is NaN, not the zeros of a row that sees nothing."""
    args = make(1, 160, 160, H, H, D, dtype, seed=58)
    args[0][..., 5] = -1.0 - args[0][..., 5].abs()
    args[1][:, 0, :, 5] = args[1][:, 59, :, 5] = math.inf
    out = pattern(q2d, args, **MASKS[name])[0]
    assert torch.isnan(out[:, 0]).all() and torch.isfinite(out[:, 1]).all()
    if name == "documents":
        assert not out[:, 50:59].any() and torch.isnan(out[:, 59]).all()


def test_more_queries_than_keys_see_nothing(q2d):
    """Rows before the first key, with and without a prefix."""
    q, k, v, _ = make(1, 100, 40, 2, 2, 64, torch.bfloat16, seed=59)
    out, lse = q2d.q2d_attention_fwd(q, k, v)
    assert not out[:, :60].any() and bool((lse[:, :, :60] == -math.inf).all()) and torch.isfinite(lse[:, :, 60:]).all()
    out, lse = q2d.q2d_attention_fwd(q, k, v, window=7)
    assert not out[:, :60].any() and bool((lse[:, :, :60] == -math.inf).all()) and torch.isfinite(lse[:, :, 60:]).all()
    for mask in (dict(prefix=torch.tensor([3], dtype=torch.int32).cuda()), dict(causal=False)):
        assert torch.isfinite(q2d.q2d_attention_fwd(q, k, v, **mask)[1]).all()
    lse = q2d.q2d_attention_fwd(q, k, v, causal=False, window=20)[1]      # |p - j| < 20: from position -19 on
    assert bool((lse[:, :, :41] == -math.inf).all()) and torch.isfinite(lse[:, :, 41:]).all()
