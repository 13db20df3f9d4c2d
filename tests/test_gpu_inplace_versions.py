"""Tensors that the norm and the clipping write in place count as modified: a backward pass that still
needs the old values is refused by autograd, as behind torch's own operators in place."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


CALLS = {
    "h": lambda q, t: q.q2d_rmsnorm_fwd(t["x"], t["w"], residual=t["r"], h=t["x"]),
    "h, residual": lambda q, t: q.q2d_rmsnorm_fwd(t["x"], t["w"], residual=t["r"], h=t["r"]),
    "y": lambda q, t: q.q2d_rmsnorm_fwd(t["x"], t["w"], y=t["y"]),
    "rstd": lambda q, t: q.q2d_rmsnorm_fwd(t["x"], t["w"], rstd=t["s"]),
    "operands": lambda q, t: q.q2d_rmsnorm_quantize(t["x"], t["w"], residual=t["r"], h=t["x"], rstd=t["s"]),
    "dx": lambda q, t: q.q2d_rmsnorm_bwd(t["y"], t["x"], t["w"], t["s"], dh=t["r"], dx=t["r"], dw=t["v"]),
    "clip": lambda q, t: q.q2d_clip_grads([t["x"], t["w"]], 1e-3),
    "clip, out": lambda q, t: q.q2d_clip_grads([t["x"], t["w"]], 1e-3, out=[t["y"], t["v"]]),
    "norm": lambda q, t: q.q2d_grad_norm([t["x"]], norm=t["n"]),
}
WRITTEN = {"h": "x", "h, residual": "r", "y": "y", "rstd": "s", "operands": "xs", "dx": "rv", "clip": "xw", "clip, out": "yv", "norm": "n"}


@pytest.mark.parametrize("call", CALLS)
def test_written_tensors_count_as_modified(q2d, call):
    g = torch.Generator().manual_seed(1)
    t = {k: torch.randn(s, generator=g).to(DEV) for k, s in
         dict(x=(6, 64), r=(6, 64), y=(6, 64), w=(64,), v=(64,), s=(6,), n=()).items()}
    before = {k: a._version for k, a in t.items()}
    CALLS[call](q2d, t)
    for k, a in t.items():
        assert (a._version > before[k]) == (k in WRITTEN[call]), k
    # tensors of inference mode have no counter
    with torch.inference_mode():
        CALLS[call](q2d, {k: a.clone() for k, a in t.items()})


def test_a_backward_pass_notices(q2d):
    for dt in (F32, BF16):
        x = torch.randn((6, 64), device=DEV, dtype=dt).requires_grad_()
        a = x * 2
        b = (a * a).sum()
        with torch.no_grad():
            q2d.q2d_rmsnorm_fwd(a, torch.ones(64, device=DEV), residual=torch.ones_like(a), h=a)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            b.backward()
        a = x * 2
        b = (a * a).sum()
        with torch.no_grad():
            q2d.q2d_clip_grads([a], 1e-3)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            b.backward()
