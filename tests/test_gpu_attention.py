"""Attention over whole sequences, forward and backward, against the definition in 64 bits.

Tolerances, from the types alone (u = 2^-8 for bfloat16's and 2^-24 for float32's relative
rounding, U = 2^-24 for the float32 arithmetic of both):

* out = sum_j P_j v_j with sum P = 1.  Each P_j is rounded (u) and out is rounded (u):
  |error| <= 2 u max_j |v_j| + A, where A covers the scores: a score of size at most s is
  off by about (dim + 4) U s, so that P is off by the same factor, and an exp2 argument by
  a few U of its size.  With |s| <= 40 in these tests, A <= 2^-24 * (128 + 64) * 40 < 2^-11
  relative at worst, and typically sqrt(dim) in place of dim; 2^-16 is taken (float32).
* The gradients sum products of rounded factors: dV = P^T dO, dQ = dS K, dK = dS^T Q, with dS
  = P (dP - delta).  delta is formed from the rounded out, |error| <= u sum |dO| |out|.  The
  sums of absolute values are formed beside the reference and the bound is 4 u of them
  (factor rounding, delta, final rounding, one to spare) plus the same A.
"""
import math

import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def make(B, Lq, Lk, Hq, Hkv, D, dtype, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    t = [torch.randn(s, generator=g) * spread for s in ((B, Lq, Hq, D), (B, Lk, Hkv, D), (B, Lk, Hkv, D), (B, Lq, Hq, D))]
    return [x.to(dtype).cuda() for x in t]


def limits(q, k, v, dout, mask, dtype):
    """Elementwise bounds of out, dq, dk, dv: the sums of absolute values of the definition."""
    c = lambda t: t.detach().cpu().double()
    q, k, v, dout = c(q), c(k), c(v), c(dout)
    B, Lq, Hq, D = q.shape
    Lk, Hkv = k.shape[1], k.shape[2]
    out, lse = ref.attention(q, k, v, **mask)
    u = U[dtype]
    A = 2.0 ** -16
    scale = mask.get("scale") or D ** -0.5
    lo, lq, lk, lv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b in range(B):
        ok = ref.seen(Lq, Lk, mask.get("causal", True), mask.get("window", 0),
                      None if mask.get("documents") is None else mask["documents"][b].cpu(),
                      0 if mask.get("prefix") is None else int(mask["prefix"][b]))
        for h in range(Hq):
            g = h // (Hq // Hkv)
            m2 = {n: x for n, x in mask.items() if n not in ("documents", "prefix", "slopes")}
            x = scale * (q[b, :, h] @ k[b, :, g].T)
            if m2.get("softcap"):
                x = m2["softcap"] * torch.tanh(x / m2["softcap"])
            if mask.get("slopes") is not None:
                x = x - float(mask["slopes"][h]) * (torch.arange(Lk - Lq, Lk)[:, None] - torch.arange(Lk)[None, :]).abs()
            P = torch.where(ok, torch.exp(x - torch.where(torch.isinf(lse[b, h]), 0.0, lse[b, h])[:, None]), 0.0)
            aV, aG = v[b, :, g].abs(), dout[b, :, h].abs()
            dP = torch.where(ok, aG @ aV.T, 0.0)
            dl = (aG * (P @ aV)).sum(1, keepdim=True)
            dS = torch.where(ok, P * (dP + dl), 0.0)
            lo[b, :, h] = (2 * u + A) * (P @ aV)
            lq[b, :, h] = (4 * u + A) * scale * (dS @ k[b, :, g].abs())
            lk[b, :, g] += (4 * u + A) * scale * (dS.T @ q[b, :, h].abs())
            lv[b, :, g] += (4 * u + A) * (P.T @ aG)
    return lo, lq, lk, lv


def check(q2d, q, k, v, dout, **mask):
    dtype = q.dtype
    dev = {n: (t.cuda() if isinstance(t, torch.Tensor) else t) for n, t in mask.items()}
    want = ref.attention(q, k, v, dout, **mask)
    bound = limits(q, k, v, dout, mask, dtype)
    out, lse = q2d.q2d_attention_fwd(q, k, v, **dev)
    grads = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, **dev)
    torch.cuda.synchronize()
    empty = torch.isinf(want[1])
    assert torch.equal(torch.isinf(lse.cpu()), empty)
    err = (lse.cpu().double() - want[1])[~empty].abs()
    assert err.numel() == 0 or float(err.max()) <= 2.0 ** -14, float(err.max())
    assert not out.cpu()[empty.transpose(1, 2)].any()
    for name, got, w, lim in zip(("out", "dq", "dk", "dv"), (out,) + tuple(grads), (want[0],) + want[2:], bound):
        e = (got.cpu().double() - w).abs()
        bad = e - lim - 1e-30
        good = bool((bad <= 0).all())
        assert good, "%s: error %.3g where %.3g is allowed" % (
            name, float(e.flatten()[bad.argmax()]), float(lim.flatten()[bad.argmax()]))
    return out, lse, grads


SHAPES = [
    # B, Lq, Lk, Hq, Hkv, D
    (1, 1, 1, 1, 1, 8),
    (2, 33, 33, 2, 1, 64),
    (1, 128, 128, 4, 4, 64),
    (1, 200, 200, 4, 2, 128),
    (2, 1, 300, 6, 2, 128),
    (1, 130, 321, 3, 1, 72),
    (1, 300, 65, 2, 2, 96),        # more queries than keys: the first see nothing under causal order
    (3, 65, 64, 7, 1, 40),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(q2d, shape, causal, dtype):
    check(q2d, *make(*shape, dtype), causal=causal)


MASKS = {
    "cap": dict(softcap=2.0),
    "cap_full": dict(softcap=30.0, causal=False),
    "window": dict(window=37),
    "window_1": dict(window=1),
    "window_full": dict(window=50, causal=False),
    "scale": dict(scale=0.31),
    "slopes": dict(slopes=torch.tensor([0.5, 0.03, 0.0, -0.01])),
    "slopes_full": dict(slopes=torch.tensor([0.5, 0.03, 0.2, 0.01]), causal=False),
    "prefix": dict(prefix=torch.tensor([100, 0], dtype=torch.int32)),
    "prefix_wide": dict(prefix=torch.tensor([10 ** 6, -5], dtype=torch.int32), window=20),
    "documents": dict(documents=torch.tensor([[0] * 70 + [1] * 1 + [2] * 129 + [-1] * 50, [5] * 250], dtype=torch.int32)),
    "documents_mixed": dict(documents=torch.tensor([[i % 3 for i in range(250)], [7 - i // 40 for i in range(250)]],
                                                   dtype=torch.int32), causal=False),
    "documents_none": dict(documents=torch.full((2, 250), -1, dtype=torch.int32)),
    "documents_prefix": dict(documents=torch.tensor([[0] * 120 + [1] * 130, [3] * 60 + [-2] * 30 + [4] * 160], dtype=torch.int32),
                             prefix=torch.tensor([150, 40], dtype=torch.int32), window=33),
    "all": dict(documents=torch.tensor([[0] * 120 + [1] * 130, [3] * 60 + [-2] * 30 + [4] * 160], dtype=torch.int32),
                softcap=5.0, slopes=torch.tensor([0.5, 0.03, 0.2, 0.01])),
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", sorted(MASKS))
def test_masks(q2d, name, D, dtype):
    check(q2d, *make(2, 250, 250, 4, 2, D, dtype, seed=3), **MASKS[name])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("name", ["cap", "slopes", "window_full", "prefix_wide", "documents", "documents_prefix", "all"])
def test_masks_of_many_heads(q2d, name, D, dtype):
    """The kernels whose workgroups own 128 rows: as many heads as give each compute unit one."""
    mask = dict(MASKS[name])
    if "slopes" in mask:
        mask["slopes"] = mask["slopes"].repeat(16)
    check(q2d, *make(2, 250, 250, 64, 64, D, dtype, seed=12), **mask)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(4, 140, 140, 64, 32, 72), (8, 64, 300, 32, 32, 128), (4, 300, 65, 32, 32, 40)], ids=str)
def test_shapes_of_many_heads(q2d, shape, dtype):
    check(q2d, *make(*shape, dtype, seed=13))


@pytest.mark.parametrize("Lq", [1, 90])
@pytest.mark.parametrize("name", ["documents", "documents_prefix", "prefix", "window", "slopes"])
def test_masks_of_last_queries(q2d, name, Lq):
    check(q2d, *make(2, Lq, 250, 4, 2, 64, torch.bfloat16, seed=4), **MASKS[name])


def test_documents_before_the_first_key(q2d):
    """More queries than keys: positions below zero belong to no document."""
    check(q2d, *make(1, 100, 40, 2, 2, 64, torch.bfloat16), documents=torch.zeros((1, 40), dtype=torch.int32), causal=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_long(q2d, dtype):
    """More than 64 key tiles, several workgroups and a ragged end."""
    check(q2d, *make(1, 257, 4500, 2, 1, 64, dtype, seed=5), causal=True)
    check(q2d, *make(1, 4500, 4500, 1, 1, 128, dtype, seed=6), window=300, prefix=torch.tensor([65], dtype=torch.int32))


def test_large_scores(q2d):
    """Scores whose exponentials overflow without the running maximum."""
    q, k, v, dout = make(1, 150, 150, 2, 2, 64, torch.float32, seed=7)
    out, lse = q2d.q2d_attention_fwd(q * 40, k * 40, v)
    want = ref.attention(q * 40, k * 40, v)
    # scores of up to about 1e5: each is off by up to its own float32 rounding
    assert torch.isfinite(out).all() and float((lse.cpu() - want[1]).abs().max() / want[1].abs().max()) < 2.0 ** -20


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fill", [math.inf, math.nan])
@pytest.mark.parametrize("B,H", [(1, 2), (2, 64)], ids=["few heads", "many heads"])
def test_unseen_non_finite(q2d, B, H, fill, D, dtype):
    """Infinities and NaN in padding, and in keys that only later queries see."""
    L = 150
    q, k, v, dout = make(B, L, L, H, H, D, dtype, seed=8)
    docs = torch.tensor([[0] * 60 + [-1] * 20 + [1] * 70] * B, dtype=torch.int32)
    clean = check(q2d, q, k, v, dout, documents=docs)
    bad = [t.clone() for t in (q, k, v, dout)]
    for t in bad:
        t[:, 60:80] = fill
    out, lse = q2d.q2d_attention_fwd(*bad[:3], documents=docs.cuda())
    grads = q2d.q2d_attention_bwd(bad[3], *bad[:3], out, lse, documents=docs.cuda())
    # the sums skip what is not seen: equal up to the order of the additions
    for x, y in zip((out,) + tuple(grads), (clean[0],) + tuple(clean[2])):
        assert torch.isfinite(x).all()
        assert float((x.float() - y.float()).abs().max()) <= 8 * U[dtype] * float(y.float().abs().max())
    # one value of one key: rows before it keep their results, rows from it on take its value
    v2 = v.clone()
    v2[:, 100, :, 3] = fill
    a = q2d.q2d_attention_fwd(q, k, v)[0]
    b = q2d.q2d_attention_fwd(q, k, v2)[0]
    assert torch.isfinite(b[:, :100]).all()
    assert float((a[:, :100].float() - b[:, :100].float()).abs().max()) <= 8 * U[dtype] * float(v.float().abs().max())
    assert not torch.isfinite(b[:, 100:, :, 3]).any()
    other = [d for d in range(D) if d != 3]
    assert torch.isfinite(b[:, 100:, :, other]).all()


def test_views_and_streams(q2d):
    """Slices of a fused projection, head-major memory, broadcast keys, another stream."""
    g = torch.Generator().manual_seed(9)
    x = torch.randn((2, 90, 8, 64), generator=g).to(torch.bfloat16).cuda()
    dout = torch.randn((2, 90, 4, 64), generator=g).to(torch.bfloat16).cuda()
    q, k, v = x[:, :, :4], x[:, :, 4:6], x[:, :, 6:]
    base = check(q2d, q, k, v, dout)
    hm = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, dout)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = torch.zeros((2, 4, 90, 64), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        lse = q2d.q2d_attention_fwd(*hm[:3], out=out)[1]
        grads = q2d.q2d_attention_bwd(hm[3], *hm[:3], out, lse)
    s.synchronize()
    assert torch.equal(out, base[0])
    for a, b in zip(grads, base[2]):
        assert torch.equal(a, b)
    kb, vb = k[:1, :, :1].expand(2, 90, 4, 64), v[:1, :, :1].expand(2, 90, 4, 64)
    check(q2d, q, kb, vb, dout)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_long_strides(q2d, dtype):
    """Rows 2^22 - 8 elements apart: offsets within a tile of 128 rows pass 2^31 bytes, and those
    of the whole tensor 2^32."""
    step, L = 2 ** 22 - 8, 150
    q, k, v, dout = make(1, L, L, 2, 1, 64, dtype, seed=14)
    far = torch.empty((L - 1) * step + 2048, dtype=dtype, device="cuda")
    args = []
    for i, t in enumerate((q, k, v, dout)):
        w = far.as_strided(t.shape, (0, step, 64, 1), 256 * i)
        w.copy_(t)
        args.append(w)
    base, got = check(q2d, q, k, v, dout), check(q2d, *args)
    assert torch.equal(base[0], got[0]) and all(torch.equal(a, b) for a, b in zip(base[2], got[2]))


def test_same_results_each_time(q2d):
    args = make(2, 300, 300, 8, 2, 128, torch.bfloat16, seed=10)
    first = check(q2d, *args, softcap=20.0)
    for _ in range(3):
        out, lse = q2d.q2d_attention_fwd(*args[:3], softcap=20.0)
        grads = q2d.q2d_attention_bwd(args[3], *args[:3], out, lse, softcap=20.0)
        assert torch.equal(out, first[0]) and all(torch.equal(a, b) for a, b in zip(grads, first[2]))


def test_gradients_against_differences(q2d):
    """Directional differences of the float32 forward pass.  Along a direction d of step t the
    central difference of the loss is off by t^2 |L'''| / 6 (taken as t^2 of the first
    derivative's scale) and by the forward rounding 2^-22 sum |dout| |out| over t."""
    q, k, v, dout = make(1, 40, 40, 2, 1, 64, torch.float32, seed=11)
    mask = dict(softcap=4.0, slopes=torch.tensor([0.1, 0.02]).cuda())
    out, lse = q2d.q2d_attention_fwd(q, k, v, **mask)
    grads = q2d.q2d_attention_bwd(dout, q, k, v, out, lse, **mask)
    loss = lambda a: float((q2d.q2d_attention_fwd(*a, **mask)[0].double() * dout.double()).sum())
    t = 2.0 ** -7
    noise = 2.0 ** -22 * float((dout.abs() * out.abs()).sum()) / t
    for i, g in enumerate(grads):
        d = torch.randn(g.shape, generator=torch.Generator().manual_seed(i)).cuda()
        plus, minus = [list((q, k, v)) for _ in range(2)]
        plus[i], minus[i] = plus[i] + t * d, minus[i] - t * d
        got = (loss(plus) - loss(minus)) / (2 * t)
        want = float((g.double() * d.double()).sum())
        scale = float(g.double().norm() * d.double().norm())
        assert abs(got - want) <= 16 * t * t * scale + noise, (i, got, want)


def test_refusals(q2d):
    q, k, v, dout = make(1, 32, 32, 4, 2, 64, torch.bfloat16)
    F = q2d.q2d_attention_fwd
    bad = [
        lambda: F(q.half(), k.half(), v.half()),
        lambda: F(q, k.float(), v),
        lambda: F(q[0], k[0], v[0]),
        lambda: F(q[..., :12], k[..., :12], v[..., :12]),              # dim not a multiple of 8
        lambda: F(q[:, :, :3], k, v),                                  # heads
        lambda: F(q, k, v[:, :31]),
        lambda: F(q, k, v, scale=0.0),
        lambda: F(q, k, v, scale=math.nan),
        lambda: F(q, k, v, softcap=-1.0),
        lambda: F(q, k, v, window=-1),
        lambda: F(q[..., 4:36], k[..., 4:36], v[..., 4:36]),           # rows off 16 bytes
        lambda: F(q.transpose(1, 3), k, v),
        lambda: F(q, k, v, slopes=torch.zeros(3, device="cuda")),
        lambda: F(q, k, v, documents=torch.zeros((1, 31), dtype=torch.int32, device="cuda")),
        lambda: F(q, k, v, documents=torch.zeros((1, 32), dtype=torch.int64, device="cuda")),
        lambda: F(q, k, v, prefix=torch.zeros(1, dtype=torch.int32)),
        lambda: F(q.cpu(), k.cpu(), v.cpu()),
        lambda: F(q, k, v, out=q[:, :, :1].expand(1, 32, 4, 64)),      # an output whose rows share memory
        lambda: F(*[torch.zeros((1, 8, 1, 136), dtype=torch.bfloat16, device="cuda")] * 3),
        lambda: q2d.q2d_attention_bwd(dout, q, k, v, q, None),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(q2d.Q2DError):
            f()
            raise AssertionError("call %d was accepted" % i)
