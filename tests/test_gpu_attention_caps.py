"""Caps of any size.  A cap far above the scores leaves them as they are; an error of tanh that
does not shrink with its argument would be multiplied by the cap.  Tolerances: those of the other
attention tests, whose allowance for the scores (2^-16) takes a relative error of 2^-22 of scores
up to 40."""
import pytest
import torch

from test_gpu_attention import check, make, q2d  # noqa: F401  (q2d: the fixture)
from test_gpu_kv_cache import attend, filled

pytestmark = pytest.mark.gpu

CAPS = [1.0, 50.0, 64.0, 65.0, 300.0, 1e4, 1e7, 1e12]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,H", [(64, 2), (64, 128), (96, 2), (128, 2), (128, 128)])
@pytest.mark.parametrize("cap", CAPS)
def test_whole_sequences(q2d, cap, D, H, dtype):
    """Scores of up to about 20; few heads and as many as give every compute unit a workgroup."""
    check(q2d, *make(1, 150, 150, H, H, D, dtype, seed=31, spread=2.0), softcap=cap)


@pytest.mark.parametrize("cap", [300.0, 1e7])
@pytest.mark.parametrize("D", [64, 128])
def test_with_distance_bias(q2d, cap, D):
    check(q2d, *make(1, 150, 150, 2, 2, D, torch.bfloat16, seed=32), softcap=cap, slopes=torch.tensor([0.3, 0.01]))


@pytest.mark.parametrize("take", ["decode", "prompt"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("cap", CAPS)
def test_over_the_cache(q2d, cap, dim, take):
    p = filled(q2d, [300, 65, 150, 64], 2, dim, seed=33, spread=2.0)
    attend(q2d, p, [1] * 4 if take == "decode" else [290, 65, 33, 64], 4, softcap=cap)


def test_scores_around_the_cap(q2d):
    """Scores from far below to far above a cap of 100: lse follows the definition to 2^-20 of the
    cap (float32 scores: a few units in their last place)."""
    import attention_ref as ref
    q, k, v, _ = make(1, 200, 200, 2, 2, 64, torch.bfloat16, seed=34)
    q = q * torch.logspace(-4, 2, 200).to(torch.bfloat16).cuda()[None, :, None, None]
    lse = q2d.q2d_attention_fwd(q, k, v, softcap=100.0)[1]
    want = ref.attention(q, k, v, softcap=100.0)[1]
    assert float((lse.cpu().double() - want).abs().max()) <= 100.0 * 2.0 ** -20
