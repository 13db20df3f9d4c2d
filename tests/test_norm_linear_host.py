"""Q2DNormLinear's parameters, which need no GPU."""
import torch


def test_reset_parameters():
    """Back to a fresh layer: the linear weight drawn anew, the norm's weight one."""
    from paper_2607_24953_amd.autograd import Q2DNormLinear
    for dtype in (torch.float32, torch.bfloat16):
        torch.manual_seed(0)
        layer = Q2DNormLinear(64, 32, seed=1, dtype=dtype)
        fresh = {k: v.clone() for k, v in layer.state_dict().items()}
        with torch.no_grad():
            for p in layer.parameters():
                p.mul_(3).add_(1)
        torch.manual_seed(0)
        layer.reset_parameters()
        assert set(fresh) == {"weight", "norm_weight"} and all(torch.equal(v, fresh[k]) for k, v in layer.state_dict().items())
        assert bool((layer.norm_weight == 1).all()) and layer.norm_weight.dtype == dtype
