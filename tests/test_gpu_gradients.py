"""The gradients' norm and clipping against 64 bits."""
import pytest
import torch

import norm_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def make(sizes, dtypes, scale=1e-3, seed=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        buf = torch.zeros(n + shift, dtype=dtypes[i % len(dtypes)], device=DEV)
        buf[shift:] = (torch.randn(n, generator=g) * scale).to(buf.dtype)
        out.append(buf[shift:])
    return out


SETS = [[1], [7], [4096], [1, 2, 3, 5, 8, 13], [16384], [16385, 16383, 1], [0, 5, 0], [100003, 9, 70000], [257] * 128,
        [33] * 129, [1000 + i for i in range(300)], [4_000_001, 3], [12] * 3000]


@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%dx%d" % (len(s), s[0]))
@pytest.mark.parametrize("dtypes", [(F32,), (BF16,), (F32, BF16)], ids=str)
@pytest.mark.parametrize("max_norm", [1e-4, 1e9])
def test_clip(q2d, sizes, dtypes, max_norm):
    for shift in (0, 1, 3):
        t = make(sizes, dtypes, shift=shift)
        norm, want = ref.clip(t, max_norm)
        got = q2d.q2d_grad_norm(t)
        assert got.dtype == F32 and got.shape == () and abs(float(got) - float(norm)) <= 2.0 ** -24 * float(norm) * (1 + 1e-9)
        out = make(sizes, dtypes, seed=1, shift=(shift + 1) % 3)
        keep = [x.clone() for x in t]
        assert torch.equal(q2d.q2d_clip_grads(t, max_norm, out=out), got)
        assert all(torch.equal(a, b) for a, b in zip(t, keep))
        assert all(torch.equal(a.cpu(), b) for a, b in zip(out, want))
        assert torch.equal(q2d.q2d_clip_grads(t, max_norm), got)
        assert all(torch.equal(a.cpu(), b) for a, b in zip(t, want))


def test_given_norm(q2d):
    t = make([5000, 33], (F32, BF16))
    given = torch.tensor(2.0, device=DEV)
    want = [(x.float() * 0.25).to(x.dtype) for x in t]
    assert q2d.q2d_clip_grads(t, 0.5, norm=given) is given
    assert all(torch.equal(a, b) for a, b in zip(t, want))
    q2d.q2d_clip_grads(t, 2.5, norm=given)
    assert all(torch.equal(a, b) for a, b in zip(t, want))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_not_finite(q2d, bad, dtype):
    """The norm says so, and the values stay as they are."""
    t = make([300, 70001], (dtype,))
    t[1][70000] = bad
    keep, out = [x.clone() for x in t], make([300, 70001], (dtype,), seed=4)
    norm = q2d.q2d_clip_grads(t, 1e-3, out=out)
    assert not bool(norm.isfinite()) and bool(norm.isnan()) == (bad != bad)
    q2d.q2d_clip_grads(t, 1e-3)
    for x in (t, out):
        assert all(torch.equal(a.view(torch.int16 if dtype == BF16 else torch.int32), b.view(torch.int16 if dtype == BF16 else torch.int32))
                   for a, b in zip(x, keep))


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-22, 1e18, 1e30])
def test_any_size(q2d, scale):
    """Squares that leave float32's range."""
    t = make([5000, 3], (F32,), scale)
    norm, want = ref.clip(t, scale)
    assert abs(float(q2d.q2d_grad_norm(t)) - float(norm)) <= 2.0 ** -24 * float(norm) * (1 + 1e-9) + 2.0 ** -149
    q2d.q2d_clip_grads(t, scale)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(t, want))


def test_bound_of_zero_and_no_elements(q2d):
    t = make([0, 0], (F32,))
    assert float(q2d.q2d_grad_norm(t)) == 0 and float(q2d.q2d_clip_grads(t, 1.0)) == 0
    z = [torch.zeros(100, device=DEV)]
    assert float(q2d.q2d_clip_grads(z, 0.0)) == 0
    t = make([50], (F32,))
    q2d.q2d_clip_grads(t, 0.0)
    assert float(t[0].abs().max()) == 0


def test_orders_of_the_dimensions(q2d):
    """Transposed tensors have no gaps either."""
    a = make([600], (F32,))[0].view(20, 30)
    b = make([24], (BF16,), seed=2)[0].view(2, 3, 4).permute(2, 0, 1)
    norm, _ = ref.clip([a, b], 1.0)
    t = [a.t(), b]
    want = [x.float() * float((1e-3 / norm).float()) for x in t]
    q2d.q2d_clip_grads(t, 1e-3)
    assert torch.equal(t[0], want[0]) and torch.equal(t[1], want[1].to(BF16))


def test_refused_lists(q2d):
    t = make([100, 50], (F32,))
    for bad in ([], [t[0], t[0]], [t[0], t[0][10:20]], [t[0][::2]], [t[0], t[1].cpu()], [t[0].double()], [t[0].view(10, 10)[:, :5]],
                [t[0].expand(3, 100)], [None], [t[0], None]):
        with pytest.raises(q2d.Q2DError):
            q2d.q2d_clip_grads(bad, 1.0)
    # the same values may be counted twice, but not scaled twice
    assert abs(float(q2d.q2d_grad_norm([t[0], t[0]])) / float(q2d.q2d_grad_norm([t[0]])) - 2 ** 0.5) < 1e-6
    for kw in (dict(out=t[::-1]), dict(out=t[:1]), dict(out=[t[0], t[1].bfloat16()]), dict(out=[t[0], t[0][:50]]),
               dict(norm=torch.tensor(1.0)), dict(norm=torch.tensor(1.0, device=DEV).double()), dict(norm=torch.ones(2, device=DEV))):
        with pytest.raises(q2d.Q2DError):
            q2d.q2d_clip_grads(t, 1.0, **kw)
    for bad in (-1.0, float("nan"), float("inf")):
        with pytest.raises(q2d.Q2DError):
            q2d.q2d_clip_grads(t, bad)


def test_far_elements(q2d):
    """A tensor of more than 2^31 elements."""
    n = (1 << 31) + 5
    t = [torch.zeros(n, dtype=BF16, device=DEV)]
    t[0][n - 3:] = 4.0
    norm = q2d.q2d_clip_grads(t, 3.0)
    assert abs(float(norm) - 48 ** 0.5) < 1e-6
    want = torch.tensor(4.0 * torch.tensor(3 / 48 ** 0.5, dtype=torch.float64).float().item()).to(BF16)
    assert bool((t[0][n - 3:].cpu() == want).all()) and float(t[0][:n - 3].abs().max()) == 0
