"""Q2DNormLinear on types that the kernels do not read, taken as float32 as by Q2DLinear, and its backward
pass in parts."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F16, F32, F64, BF16 = torch.float16, torch.float32, torch.float64, torch.bfloat16


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).to(DEV)


@pytest.mark.parametrize("residual", [None, F32, BF16, F16, F64], ids=str)
@pytest.mark.parametrize("x,w", [(F16, F16), (F64, F64), (F16, F32), (BF16, F16), (F32, F64)], ids=str)
def test_other_types(x, w, residual):
    """Values and gradients are those of the layer on the float32 values, rounded to the types."""
    from paper_2607_24953_amd.autograd import Q2DNormLinear
    X = rand(5, 30, 160, dtype=x, seed=1)
    R = None if residual is None else rand(5, 30, 160, dtype=residual, seed=2)
    kind = lambda t: t if t is None or t.dtype in (F32, BF16) else t.float()
    layer = Q2DNormLinear(160, 96, seed=7, device=DEV)
    with torch.no_grad():
        layer.norm_weight += rand(160, seed=8, scale=0.2)
    layer = layer.to(w)
    plain = Q2DNormLinear(160, 96, seed=7, device=DEV)
    plain.load_state_dict({k: v.float() for k, v in layer.state_dict().items()})
    got, want = [], []
    for model, (a, b), out in ((layer, (X, R), got), (plain, (kind(X), kind(R)), want)):
        a = a.detach().requires_grad_()
        b = None if b is None else b.detach().requires_grad_()
        o = model(a, b)
        Y, H = o if b is not None else (o, None)
        dY = rand(5, 30, 96, dtype=BF16, seed=3)
        if b is None:
            Y.backward(dY)
        else:
            # (a gradient that every type holds)
            torch.autograd.backward((Y, H), (dY, rand(5, 30, 160, dtype=BF16, seed=4).to(F16).to(H.dtype)))
        out += [Y, H, a.grad, None if b is None else b.grad, model.weight.grad, model.norm_weight.grad]
    kinds = [BF16, x, x, residual, w, w]
    for i, (a, b, k) in enumerate(zip(got, want, kinds)):
        assert (a is None) == (b is None), i
        if a is not None:
            assert a.dtype == k and torch.equal(a, b.to(k)), i


def test_backward_by_the_sum_alone_first():
    """A pass through x + residual reads no operands: the pass through Y may still come."""
    from paper_2607_24953_amd.autograd import Q2DNormLinear
    dY, dH = rand(50, 96, dtype=BF16, seed=3), rand(50, 160, seed=4)
    grads = []
    for apart in (True, False):
        layer = Q2DNormLinear(160, 96, seed=7, device=DEV)
        with torch.no_grad():
            layer.weight.copy_(rand(96, 160, seed=5, scale=0.1))
        X, R = rand(50, 160, seed=1).requires_grad_(), rand(50, 160, seed=2).requires_grad_()
        Y, H = layer(X, R)
        if apart:
            H.backward(dH, retain_graph=True)
            assert torch.equal(X.grad, dH) and layer.weight.grad is None
            Y.backward(dY)
        else:
            torch.autograd.backward((Y, H), (dY, dH))
        grads.append([t.grad for t in (X, R, layer.weight, layer.norm_weight)])
    # (dh's addition is the last step of dx, in float32 both times)
    assert all(torch.equal(a, b) for a, b in zip(*grads))
