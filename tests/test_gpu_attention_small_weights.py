"""Keys that have small weights from all queries (a distance bias, more keys than queries):
their gradients are as exact, for their size, as others'."""
import pytest
import torch

from test_gpu_attention import check, make, q2d  # noqa: F401  (q2d: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 72, 96, 128])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
@pytest.mark.parametrize("H", [4, 64], ids=["few heads", "many heads"])
def test_far_keys(q2d, H, softcap, D, dtype):
    """Weights down to 2^-300: those above 2^-100 count (gradients below 1e-30 may be 0)."""
    slopes = torch.tensor([0.05, 0.13, 0.25, 0.5]).repeat(H // 4)
    check(q2d, *make(1, 100, 400, H, H, D, dtype, seed=91), slopes=slopes, softcap=softcap)


def test_keys_of_very_different_weights(q2d):
    """Both kinds side by side: a window of far keys next to near ones, and columns of a tile that
    see nothing."""
    slopes = torch.tensor([0.3, 0.02] * 32)
    check(q2d, *make(1, 90, 420, 64, 64, 128, torch.bfloat16, seed=92), slopes=slopes, window=300,
          prefix=torch.tensor([37], dtype=torch.int32))
