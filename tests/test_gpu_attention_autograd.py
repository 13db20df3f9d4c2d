"""What the autograd form of attention keeps between forward and backward."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def make(**kw):
    from paper_2607_24953_amd.autograd import attention
    g = torch.Generator().manual_seed(81)
    q, k, v = (torch.randn((1, 70, 2, 64), generator=g).to(torch.bfloat16).cuda().requires_grad_() for _ in range(3))
    return attention(q, k, v, **kw), (q, k, v)


@pytest.mark.parametrize("name", ["documents", "prefix", "slopes"])
def test_masks_changed_in_place(name):
    """Backward needs the masks of the forward call: a change in place is an error."""
    t = {"documents": torch.zeros((1, 70), dtype=torch.int32), "prefix": torch.zeros(1, dtype=torch.int32),
         "slopes": torch.ones(2)}[name].cuda()
    out, _ = make(**{name: t})
    out.sum().backward()
    out, _ = make(**{name: t})
    t += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_no_second_derivative():
    """The gradients are computed outside of autograd: asking for their own is an error."""
    out, inputs = make()
    grads = torch.autograd.grad(out.float().square().sum(), inputs, create_graph=True)
    with pytest.raises(RuntimeError):
        (out.float().sum() + sum(g.float().sum() for g in grads)).backward()


def test_arguments_are_refused_in_forward():
    for kw in (dict(out=None), dict(need_lse=False), dict(caual=True)):
        with pytest.raises(TypeError):
            make(**kw)


def test_gradient_off_16_bytes():
    """A gradient that is a contiguous slice at any offset (attention's output behind others in one
    tensor), and one whose rows lie 2^22 elements apart."""
    from paper_2607_24953_amd.autograd import attention
    g = torch.Generator().manual_seed(82)
    q, k, v, w = (torch.randn((1, 70, 2, 64), generator=g).to(torch.bfloat16).cuda().requires_grad_() for _ in range(4))
    want = torch.autograd.grad(attention(q, k, v), (q, k, v), w.detach())
    lead = torch.zeros(3, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    out = torch.cat((lead, attention(q, k, v).flatten()))
    got = torch.autograd.grad(out, (q, k, v), torch.cat((lead.detach(), w.detach().flatten())))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    far = torch.empty(69 * 2 ** 22 + 128, dtype=torch.bfloat16, device="cuda").as_strided((1, 70, 2, 64), (0, 2 ** 22, 64, 1))
    far.copy_(w.detach())
    got = torch.autograd.grad(attention(q, k, v), (q, k, v), far)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
