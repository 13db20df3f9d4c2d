"""The operators together: training through autograd, then prompts and single tokens out of
the cache."""
import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu


def test_autograd_matches_the_operators():
    import paper_2607_24953_amd as q2d
    from paper_2607_24953_amd.autograd import attention
    g = torch.Generator().manual_seed(0)
    x = torch.randn((2, 70, 8, 64), generator=g).to(torch.bfloat16).cuda().requires_grad_()
    slopes = torch.tensor([0.3, 0.1, 0.01, 0.0]).cuda()
    mask = dict(softcap=5.0, slopes=slopes)
    out = attention(x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], **mask)
    dout = torch.randn(out.shape, generator=g).to(torch.bfloat16).cuda()
    out.backward(dout)
    q, k, v = (t.detach() for t in (x[:, :, :4], x[:, :, 4:6], x[:, :, 6:]))
    o, lse = q2d.q2d_attention_fwd(q, k, v, **mask)
    grads = q2d.q2d_attention_bwd(dout, q, k, v, o, lse, **mask)
    assert torch.equal(out, o) and torch.equal(x.grad, torch.cat(grads, 2))
    # a gradient with broadcast strides
    out = attention(q.requires_grad_(), k, v, **mask)
    out.sum().backward()
    want = ref.attention(q, k, v, torch.ones_like(out), softcap=5.0, slopes=slopes.cpu())[2]
    # the terms of a row cancel (dout is constant): the bound of the operators' own tests, 4 u of
    # the sums of absolute values, is at most 4 u * scale * 2 * sum |v| max |k|
    u = 2.0 ** -8
    lim = 4 * u * 64 ** -0.5 * 2 * float(v.detach().float().abs().sum(-1).max()) * float(k.detach().float().abs().max())
    assert float((q.grad.cpu().double() - want).abs().max()) <= lim


def test_decoder_learns_and_answers_from_the_cache():
    """Phrases that repeat can be continued: the loss falls far below its start (log 64 = 4.2),
    and most continuations out of the 8-bit cache are right."""
    from paper_2607_24953_amd.decoder import Decoder, train
    torch.manual_seed(0)
    model = Decoder()
    losses = train(model, 300)
    assert losses[0] > 3.5 and sum(losses[-10:]) / 10 < 1.0, (losses[0], losses[-10:])
    g = torch.Generator().manual_seed(2)
    phrases = [torch.randint(64, (int(n),), generator=g) for n in torch.randint(4, 13, (16,), generator=g)]
    got = model.generate([f.repeat(3) for f in phrases], 12).cpu()
    want = torch.stack([f.repeat(8)[:12] for f in phrases])
    assert float((got == want).float().mean()) > 0.6
