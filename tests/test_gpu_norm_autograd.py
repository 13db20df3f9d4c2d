"""The norm, the linear layer behind it and the clipping in a model: autograd, streams, graphs."""
import pytest
import torch

import norm_ref as ref
from helpers import assert_same_bytes, gpu_buffers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).to(DEV)


@pytest.mark.parametrize("residual", [None, BF16, F32], ids=str)
@pytest.mark.parametrize("x", [F32, BF16], ids=str)
def test_rms_norm(q2d, x, residual):
    """Values and gradients are those of the operators, for any leading shape."""
    from paper_2607_24953_amd.autograd import rms_norm
    X, W = rand(2, 5, 3, 100, dtype=x, seed=1).requires_grad_(), (1 + rand(100, seed=2, scale=0.1)).requires_grad_()
    R = None if residual is None else rand(2, 5, 3, 100, dtype=residual, seed=3).requires_grad_()
    dy, dh = rand(2, 5, 3, 100, dtype=BF16, seed=4), rand(2, 5, 3, 100, dtype=x, seed=5)
    out = rms_norm(X, W, residual=R)
    flat = lambda t: None if t is None else t.detach().reshape(-1, 100)
    y, h, rstd = q2d.q2d_rmsnorm_fwd(flat(X), W.detach(), residual=flat(R))
    if R is None:
        assert torch.equal(flat(out), y)
        out.backward(dy)
        dx, dw = q2d.q2d_rmsnorm_bwd(flat(dy), h, W.detach(), rstd)
    else:
        assert torch.equal(flat(out[0]), y) and torch.equal(flat(out[1]), h) and out[1].dtype == x
        torch.autograd.backward(out, (dy, dh))
        dx, dw = q2d.q2d_rmsnorm_bwd(flat(dy), h, W.detach(), rstd, dh=flat(dh))
        assert torch.equal(flat(R.grad), dx.to(residual)) and R.grad.dtype == residual
    assert torch.equal(flat(X.grad), dx) and torch.equal(W.grad, dw)


def test_rms_norm_gradients_that_are_missing(q2d):
    """Only one of the two outputs used; inputs without gradients; broadcast gradients; views."""
    from paper_2607_24953_amd.autograd import rms_norm
    W = (1 + rand(64, seed=2, scale=0.1)).requires_grad_()
    X, R = rand(6, 64, seed=1).requires_grad_(), rand(6, 64, seed=3).requires_grad_()
    y, h = rms_norm(X, W, residual=R, y_dtype=F32)
    h.sum().backward()
    assert bool((X.grad == 1).all()) and bool((R.grad == 1).all()) and W.grad is None
    X.grad = R.grad = None
    y, h = rms_norm(X, W, residual=R, y_dtype=F32)
    y.sum().backward()                                      # (a gradient of stride 0)
    want, tol, want_w, tol_w = ref.backward(torch.ones(6, 64), (X + R).detach(), W.detach(),
                                            q2d.q2d_rmsnorm_fwd((X + R).detach(), W.detach())[2], None)
    assert bool(((X.grad.cpu().double() - want).abs() <= tol).all()) and torch.equal(X.grad, R.grad)
    assert bool(((W.grad.cpu().double() - want_w).abs() <= tol_w).all())
    frozen = W.detach()
    X.grad = None
    rms_norm(X, frozen, residual=R.detach())[0].float().sum().backward()
    assert X.grad is not None
    wide = rand(64, 12, seed=7).requires_grad_()
    rms_norm(wide.t(), W.detach(), y_dtype=F32).square().sum().backward()       # rows without unit stride
    assert wide.grad.shape == wide.shape and bool(wide.grad.isfinite().all())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y, h = rms_norm(X, W, residual=R)
        h.data_ptr()
        with torch.no_grad():
            W += 1
        y.sum().backward()


def test_gradients_share_no_memory(q2d):
    """Gradients of x, the residual and other tensors can be changed in place, one by one."""
    from paper_2607_24953_amd.autograd import rms_norm
    W = torch.ones(64, device=DEV)
    for use in ("y", "h", "both"):
        X, R, Z = (rand(6, 64, seed=i).requires_grad_() for i in (1, 3, 5))
        y, h = rms_norm(X, W, residual=R, y_dtype=F32)
        k = rand(6, 64, seed=9)
        (((h + Z) * k).sum() if use == "h" else (y * k).sum() if use == "y" else ((h + Z) * k).sum() + y.sum()).backward()
        grads = [t.grad for t in (X, R, Z) if t.grad is not None]
        keep = [g.clone() for g in grads]
        assert len({g.untyped_storage().data_ptr() for g in grads}) == len(grads)
        for i, g in enumerate(grads):
            g.mul_(2)
            assert all(torch.equal(a, b * (2 if j <= i else 1)) for j, (a, b) in enumerate(zip(grads, keep)))


def test_rms_norm_refusals(q2d):
    from paper_2607_24953_amd.autograd import rms_norm
    W = torch.ones(64, device=DEV)
    for x, r, w in ((rand(4, 63), None, W), (rand(4, 64), rand(64), W), (rand(4, 64), None, W[None]), (rand(4, 64).double(), None, W),
                    (rand(4, 64).half(), None, W), (rand(4, 64).cpu(), None, W), (rand(4, 64), rand(4, 64).cpu(), W)):
        with pytest.raises(q2d.Q2DError):
            rms_norm(x, w, residual=r)
    X = rand(4, 64).requires_grad_()
    g, = torch.autograd.grad(rms_norm(X, W, y_dtype=F32).square().sum(), X, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("options", [dict(), dict(activations="1d"), dict(block=64), dict(out_dtype=F32), dict(dtype=BF16)], ids=str)
@pytest.mark.parametrize("residual", [True, False])
def test_norm_linear(q2d, options, residual, monkeypatch):
    """The layer is its operators, one after the other."""
    from paper_2607_24953_amd.autograd import Q2DNormLinear
    layer = Q2DNormLinear(160, 96, device=DEV, seed=11, **options)
    with torch.no_grad():
        layer.norm_weight += rand(160, seed=8, scale=0.2).to(layer.norm_weight.dtype)
    X, R = rand(3, 50, 160, seed=9).requires_grad_(), rand(3, 50, 160, dtype=BF16, seed=10).requires_grad_() if residual else None
    out = layer(X, R)
    Y, H = out if residual else (out, None)
    flat = lambda t: None if t is None else t.detach().reshape(-1, t.shape[-1])
    fmt, block = (q2d.FP4_1D, 32) if layer.activations == "1d" else (q2d.FP4_2D, layer.block)
    nw = layer.norm_weight.detach()
    (qX,), h, rstd = q2d.q2d_rmsnorm_quantize(flat(X), nw, residual=flat(R), formats=(fmt,), block=block)
    qW = q2d.q2d_quantize(layer.weight.detach(), "rtn", block=layer.block)
    want = q2d.q2d_gemm(qX, 0, qW, 0, out_dtype=layer.out_dtype)
    assert torch.equal(flat(Y), want) and Y.dtype == layer.out_dtype and (H is None or torch.equal(flat(H), h))
    dY, dH = rand(*Y.shape, dtype=Y.dtype, seed=12), rand(3, 50, 160, seed=13)
    torch.autograd.backward([Y, H] if residual else [Y], [dY, dH] if residual else [dY])
    dy, dW, _ = q2d.q2d_linear_bwd(flat(dY), qX, qW, "sr", 11, 2, dx_dtype=dY.dtype, block=layer.block)
    dx, dw = q2d.q2d_rmsnorm_bwd(dy, h, nw, rstd, dh=flat(dH) if residual else None)
    assert torch.equal(flat(X.grad), dx) and torch.equal(layer.weight.grad, dW.to(layer.weight.dtype))
    assert torch.equal(layer.norm_weight.grad, dw.to(nw.dtype)) and (not residual or torch.equal(flat(R.grad), dx.to(BF16)))
    # evaluation writes the rowwise copies alone, with the same result
    from paper_2607_24953_amd import autograd
    seen = []
    monkeypatch.setattr(autograd, "q2d_rmsnorm_quantize",
                        lambda *a, **kw: seen.append(kw["orientations"]) or q2d.q2d_rmsnorm_quantize(*a, **kw))
    layer(X, R)
    with torch.no_grad():
        again = layer(X, R)
    assert torch.equal(again[0] if residual else again, Y) and seen == [(True, True), (True, False)]


def test_norm_linear_second_backward(q2d):
    from paper_2607_24953_amd.autograd import Q2DNormLinear
    with pytest.raises(ValueError):
        Q2DNormLinear(64, 64, mode_x="sr", device=DEV)
    layer = Q2DNormLinear(64, 64, device=DEV)
    loss = layer(rand(32, 64).requires_grad_()).float().sum()
    loss.backward(retain_graph=True)
    with pytest.raises(q2d.Q2DError):
        loss.backward()


def test_decoder_on_rms_norms(q2d):
    """It trains with clipped gradients, and answers out of the cache."""
    from paper_2607_24953_amd.decoder import Decoder, repeated_phrases, train
    torch.manual_seed(0)
    model = Decoder(norm="rms")
    losses = train(model, 3, rows=4, length=128, clip=0.05)
    assert all(x == x for x in losses)
    norm = torch.sqrt(sum(p.grad.double().square().sum() for p in model.parameters()))
    # each element is off by the factor's rounding and its own, 2^-24 each
    assert float(norm) <= 0.05 * (1 + 2.0 ** -22)
    assert all(p.grad is not None and bool(p.grad.isfinite().all()) for p in model.parameters())
    got = model.generate([torch.arange(5), torch.arange(9)], 4)
    assert got.shape == (2, 4) and int(got.min()) >= 0 and int(got.max()) < 64
    # prompts through the cache in one step and token by token: the same operators
    caches = model.caches(4)
    table = torch.arange(4, dtype=torch.int32, device=DEV).view(2, 2)
    tokens = torch.randint(64, (2, 6), device=DEV)
    lens = torch.full((2,), 6, dtype=torch.int32, device=DEV)
    whole = model.step(tokens.flatten(), caches, table, lens).view(2, 6, -1)
    assert whole.shape == (2, 6, 64) and bool(whole.isfinite().all())
    with pytest.raises(ValueError):
        Decoder(norm="batch")


def test_step_in_a_graph(q2d):
    """A norm, a layer, the loss's gradient back through both, and the clipping of all gradients,
    captured: each replay gives the eager step's bytes, with other work between."""
    T, C, N = 200, 512, 384
    X, R, W = rand(T, C, seed=1), rand(T, C, dtype=BF16, seed=2), 1 + rand(C, seed=3, scale=0.1)
    WL, dY, dh = rand(N, C, seed=4, scale=0.05), rand(T, N, dtype=BF16, seed=5, scale=1e-3), rand(T, C, seed=6, scale=1e-3)

    def step():
        (qX, q8), h, rstd = q2d.q2d_rmsnorm_quantize(X, W, residual=R, formats=(q2d.FP4_2D, q2d.MXFP8))
        qW = q2d.q2d_quantize(WL)
        Y = q2d.q2d_gemm(qX, 0, qW, 0, out_dtype=BF16)
        dy, dW, _ = q2d.q2d_linear_bwd(dY, qX, qW, "sr", 3, 2)
        dx, dw = q2d.q2d_rmsnorm_bwd(dy, h, W, rstd, dh=dh)
        norm = q2d.q2d_clip_grads([dW, dw], 1e-3)
        y = q2d.q2d_rmsnorm_fwd(dx, W, y_dtype=F32)[0]
        return [Y, h, rstd, dx, dw, dW, norm, q2d.q2d_grad_norm([dx, dw]), y] + [getattr(q, n) for q in (qX, q8) for n in
                                                                                  ("codes", "codes_t", "scales", "scales_t")]
    want = [t.clone() for t in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for _ in range(4):
        for g, out in graphs:
            for t in out:
                t.zero_()
            g.replay()
            step()                                          # eager work beside it
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(out, want)):
                assert torch.equal(a.view(torch.uint8) if a.dim() else a, b.view(torch.uint8) if b.dim() else b), i
    # new inputs in place
    X += 1
    want = [t.clone() for t in step()]
    graphs[0][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(graphs[0][1], want))


def test_backward_in_a_graph(q2d):
    """rms_norm and Q2DNormLinear with their backward pass captured: each replay gives the bytes of
    the eager pass.  (No eager output of the leaves is alive while the capture runs.)"""
    from paper_2607_24953_amd.autograd import Q2DNormLinear, rms_norm
    T, C, N = 130, 256, 192
    layer = Q2DNormLinear(C, N, mode_dy="rtn", device=DEV, dtype=F32)
    with torch.no_grad():
        layer.weight.copy_(rand(N, C, seed=1, scale=0.05))
        layer.norm_weight.copy_(1 + rand(C, seed=2, scale=0.1))
    X, R, W = rand(T, C, seed=3).requires_grad_(), rand(T, C, seed=4).requires_grad_(), (1 + rand(N, seed=5, scale=0.1)).requires_grad_()
    gy, gh = rand(T, N, seed=6), rand(T, C, seed=7)
    leaves = [X, R, W, layer.weight, layer.norm_weight]

    def step():
        Y, h = layer(X, R)
        y = rms_norm(Y, W, y_dtype=F32)
        return [y.detach(), h.detach()] + list(torch.autograd.grad((y, h), leaves, (gy, gh)))
    want = [t.clone() for t in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for _ in range(4):
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a, b), i
        _ = torch.randn(1000, device=DEV).sum().item()      # eager work between replays


def test_other_streams(q2d):
    """Calls on a stream of their own, two at once."""
    X, R, W = rand(3000, 1024, dtype=BF16, seed=1), rand(3000, 1024, dtype=BF16, seed=2), 1 + rand(1024, seed=3, scale=0.1)
    dy = rand(3000, 1024, dtype=BF16, seed=4, scale=1e-3)

    def work():
        y, h, rstd = q2d.q2d_rmsnorm_fwd(X, W, residual=R)
        (q,), h2, _ = q2d.q2d_rmsnorm_quantize(X, W, residual=R)
        dx, dw = q2d.q2d_rmsnorm_bwd(dy, h, W, rstd)
        out = [torch.empty_like(dx), torch.empty_like(dw)]
        return [y, h, rstd, h2, q.codes, q.codes_t, dx, dw, q2d.q2d_clip_grads([dx, dw], 0.1, out=out), *out]

    want = work()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    torch.cuda.synchronize()
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(work())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
