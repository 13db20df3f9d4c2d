"""The paged 8-bit key/value cache and attention over it.

Codes and scales are compared bit for bit with the host's definition.  Attention is compared
with the definition in 64 bits on the values that the codes stand for; its tolerance is that
of the forward kernel's tests: (2 u + A) sum_j P_j |v_j| with u = 2^-8 (probabilities and
output rounded to bfloat16) and A = 2^-16 for the float32 scores."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from kv_ref import Paged, decode, encode

U, A = 2.0 ** -8, 2.0 ** -16


def test_reference_codec_against_torch():
    c = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(c).view(torch.float8_e4m3fn).float().numpy()
    got = decode(c)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    x = np.concatenate((np.linspace(-448, 448, 40001), 2.0 ** np.arange(-14, 8.8, 0.01), np.arange(0, 64) * 2.0 ** -11))
    assert np.array_equal(encode(x.astype(np.float32).astype(np.float64)),
                          torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def tokens(n, heads, dim, dtype=torch.bfloat16, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn((n, heads, dim), generator=g) * spread).to(dtype).cuda() for _ in range(2)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,dim,page", [(1, 16, 32), (3, 64, 64), (2, 80, 96), (4, 128, 64), (8, 128, 256)])
def test_write_and_read(q2d, heads, dim, page, dtype):
    counts = [1, 0, 33, 100, 64, 31]
    p = Paged(q2d, len(counts), heads, dim, page)
    for step in range(3):
        p.append(*tokens(sum(counts), heads, dim, dtype, seed=step, spread=4.0 ** step), counts)
        p.check()
    # the last tokens of each sequence, and all of them
    for take in ([1, 0, 40, 7, 192, 93], [int(n) for n in p.lens()]):
        off = torch.tensor(np.concatenate(([0], np.cumsum(take))), dtype=torch.int64).cuda()
        for dt in (torch.float32, torch.bfloat16):
            k, v = q2d.q2d_kv_read(p.cache, p.table.cuda(), p.lens().cuda(), sum(take), offsets=off, out_dtype=dt)
            at = 0
            for b, n in enumerate(take):
                dk, dv = p.dense(b)
                assert torch.equal(k[at:at + n].cpu().double(), dk[len(dk) - n:])
                assert torch.equal(v[at:at + n].cpu().double(), dv[len(dv) - n:])
                at += n


@pytest.mark.gpu
def test_token_by_token(q2d):
    """Appends of one token whose magnitudes grow and shrink: earlier codes are rounded again."""
    p = Paged(q2d, 3, 2, 64, 32)
    g = torch.Generator().manual_seed(1)
    for step in range(70):
        spread = 2.0 ** torch.randint(-6, 7, (3, 1, 1), generator=g)
        k, v = [(torch.randn((3, 2, 64), generator=g) * spread).to(torch.bfloat16).cuda() for _ in range(2)]
        if step == 5:
            k[1], v[1] = 0, 0
        # one token each, with and without offsets
        if step % 2:
            p.append(k, v, [1, 1, 1])
        else:
            for b in range(3):
                for h in range(2):
                    p.k[b][h].append(k[b:b + 1, h].float().cpu().numpy())
                    p.v[b][h].append(v[b:b + 1, h].float().cpu().numpy())
            q2d.q2d_kv_write(p.cache, k, v, p.table.cuda(), p.lens().cuda())
        if step % 9 == 0 or step > 60:
            p.check()


@pytest.mark.gpu
def test_special_values(q2d):
    p = Paged(q2d, 4, 1, 32, 32)
    k, v = tokens(4 * 40, 1, 32, torch.float32, seed=2)
    k[3, 0, 5], v[45, 0, 0] = math.inf, math.nan
    k[80:120] = 0.0
    v[80:120] *= 2.0 ** -130
    k[120:160] *= 2.0 ** 120
    p.append(k, v, [40] * 4)
    p.check()
    # a NaN joins a block that has tokens, and later tokens join that block
    for step in range(2):
        k, v = tokens(4, 1, 32, torch.float32, seed=3 + step)
        if step == 0:
            k[1, 0, 31] = -math.inf
        p.append(k, v, [1] * 4)
        p.check()
    k, v = q2d.q2d_kv_read(p.cache, p.table.cuda(), p.lens().cuda(), 4 * 42)
    for b in range(4):
        for got, want in zip((k, v), p.dense(b)):
            assert np.array_equal(got[42 * b:42 * b + 42].cpu().double().numpy(), want.numpy(), equal_nan=True)


@pytest.mark.gpu
def test_strided_tokens_and_bad_tables(q2d):
    p = Paged(q2d, 2, 2, 64, 32, capacity=96)
    x = torch.randn((50, 2, 2, 64), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    p.append(x[:, 0], x[:, 1], [20, 30])
    p.check()
    before = [getattr(p.cache, n).clone() for n in ("k_codes", "v_codes_t", "k_scales", "v_scales")]
    k, v = x[:2, 0], x[:2, 1]
    # tables that name no page, lengths of nothing: nothing is written
    for table, lens in ((torch.full_like(p.table, -1), [21, 31]), (torch.full_like(p.table, p.cache.pages), [21, 31]),
                        (p.table, [0, -7])):
        q2d.q2d_kv_write(p.cache, k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    for n, t in zip(("k_codes", "v_codes_t", "k_scales", "v_scales"), before):
        assert torch.equal(getattr(p.cache, n), t)
    # more rows than the sequence has tokens: the rows before its first position are left out
    p2 = Paged(q2d, 1, 2, 64, 32, capacity=96)
    q2d.q2d_kv_write(p2.cache, x[:10, 0], x[:10, 1], p2.table.cuda(), torch.tensor([4], dtype=torch.int32).cuda())
    for h in range(2):
        p2.k[0][h].append(x[6:10, 0, h].float().cpu().numpy())
        p2.v[0][h].append(x[6:10, 1, h].float().cpu().numpy())
    p2.check()


def attend(q2d, p, take, heads_q, seed=0, wide_table=0, **mask):
    """q2d_attention_cached on the last take[b] tokens of each sequence against the definition."""
    g = torch.Generator().manual_seed(100 + seed)
    n = sum(take)
    q = torch.randn((n, heads_q, p.dim), generator=g).to(torch.bfloat16).cuda()
    off = torch.tensor(np.concatenate(([0], np.cumsum(take))), dtype=torch.int64).cuda()
    dev = {m: (t.cuda() if isinstance(t, torch.Tensor) else t) for m, t in mask.items()}
    table = p.table
    if wide_table:
        table = torch.cat((table, torch.full((table.shape[0], wide_table), -1, dtype=torch.int32)), 1)
    out = q2d.q2d_attention_cached(q, p.cache, table.cuda(), p.lens().cuda(), offsets=off, **dev)
    if len(set(take)) == 1 and n:
        same = q2d.q2d_attention_cached(q, p.cache, table.cuda(), p.lens().cuda(), **dev)
        assert torch.equal(same.view(torch.int16), out.view(torch.int16))
    at = 0
    for b, m in enumerate(take):
        if m == 0:
            continue
        k, v = p.dense(b)
        rows = q[at:at + m][None]
        one = dict(mask)
        if one.get("prefix") is not None:
            one["prefix"] = one["prefix"][b:b + 1]
        want, lse = ref.attention(rows, k[None], v[None], **one)
        bound = (2 * U + A) * ref.attention(rows, k[None], v[None].abs(), **one)[0]
        got = out[at:at + m].cpu().double()[None]
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan), (b, "NaN")
        err = torch.where(nan, 0.0, (got - want).abs() - bound.nan_to_num() - 1e-30)
        good = bool((err <= 0).all())
        assert good, (b, float(err.max()))
        at += m
    return q, out


def filled(q2d, counts, heads, dim, page=64, capacity=512, seed=0, spread=1.0):
    p = Paged(q2d, len(counts), heads, dim, page, capacity, seed)
    p.append(*tokens(sum(counts), heads, dim, seed=seed, spread=spread), counts)
    return p


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [16, 64, 96, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (1, 7), (2, 16), (1, 40)])
def test_decode(q2d, heads, group, dim):
    counts = [1, 32, 33, 64, 65, 130, 257, 300]
    p = filled(q2d, counts, heads, dim)
    attend(q2d, p, [1] * len(counts), heads * group, wide_table=0)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [32, 64, 160])
@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_and_mixed(q2d, dim, page):
    counts = [5, 300, 128, 1, 200, 77]
    p = filled(q2d, counts, 2, dim, page)
    attend(q2d, p, counts, 8)
    attend(q2d, p, [5, 100, 0, 1, 199, 1], 8, seed=1)
    attend(q2d, p, [3] * 5 + [64], 2, seed=2)
    attend(q2d, p, [0, 0, 0, 1, 0, 0], 2, seed=3)


MASKS = {
    "cap": dict(softcap=2.0),
    "window": dict(window=40),
    "window_1": dict(window=1),
    "scale": dict(scale=0.4),
    "slopes": dict(slopes=torch.tensor([0.5, 0.02, 0.0, -0.01])),
    "prefix": dict(prefix=torch.tensor([100, 0, 1000, 17], dtype=torch.int32)),
    "prefix_window": dict(prefix=torch.tensor([10, 0, 20, -4], dtype=torch.int32), window=33),
    "all": dict(prefix=torch.tensor([10, 0, 20, 64], dtype=torch.int32), window=50, softcap=3.0,
                slopes=torch.tensor([0.5, 0.02, 0.1, 0.01])),
}


@pytest.mark.gpu
@pytest.mark.parametrize("take", ["decode", "prompt"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("name", sorted(MASKS))
def test_masks(q2d, name, dim, take):
    counts = [300, 65, 150, 64]
    p = filled(q2d, counts, 2, dim, seed=5)
    attend(q2d, p, [1] * 4 if take == "decode" else [290, 65, 33, 64], 4, **MASKS[name])


@pytest.mark.gpu
def test_long_contexts(q2d):
    """Many splits, a table wider than the sequences, and few and many heads."""
    counts = [5000, 3, 2111]
    p = filled(q2d, counts, 1, 128, 64, 5056, seed=6)
    attend(q2d, p, [1, 1, 1], 4, wide_table=0)
    attend(q2d, p, [1, 1, 1], 4, wide_table=300)
    attend(q2d, p, [70, 3, 1], 4, wide_table=10)
    attend(q2d, p, [1, 1, 1], 1, window=700, softcap=10.0)


@pytest.mark.gpu
def test_more_sequences_than_a_wave(q2d):
    counts = [1 + (i * 7) % 70 for i in range(150)]
    p = filled(q2d, counts, 1, 64, 32, 96, seed=7)
    p.check()
    attend(q2d, p, [1] * 150, 2)
    attend(q2d, p, [min(n, i % 5) for i, n in enumerate(counts)], 2)


@pytest.mark.gpu
def test_blocks_with_nan(q2d):
    """A NaN is met by the queries that see its block, and by no other."""
    p = Paged(q2d, 2, 1, 64, 32)
    k, v = tokens(300, 1, 64, seed=8)
    k[100, 0, 3], v[290, 0, 7] = math.nan, math.inf         # sequence 0: block 3; sequence 1: block 4
    p.append(k, v, [150, 150])
    attend(q2d, p, [150, 150], 2)
    attend(q2d, p, [150, 150], 2, window=20)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("take", [1, 150])
def test_blocks_with_nan_of_vanishing_weight(q2d, take, dim):
    """Values that are NaN reach a query that sees them also where their weight underflows."""
    p = Paged(q2d, 1, 1, dim, 32)
    k, v = tokens(150, 1, dim, seed=12, spread=80.0)
    k[96:128], v[100, 0, 3] = 0.0, math.nan                 # scores of 0 beside ones of some hundreds
    p.append(k, v, [150])
    q = torch.randn((take, 4, dim), generator=torch.Generator().manual_seed(13)).to(torch.bfloat16).cuda()
    out = q2d.q2d_attention_cached(q, p.cache, p.table.cuda(), p.lens().cuda())
    sees = torch.arange(150 - take, 150).cuda() >= 96
    assert torch.equal(torch.isnan(out), sees[:, None, None].expand_as(out))


@pytest.mark.gpu
def test_missing_pages(q2d):
    """A table entry that names no page: its tokens are not seen."""
    p = filled(q2d, [200], 1, 64, 64, 256)
    q = torch.randn((1, 2, 64), generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).cuda()
    k, v = p.dense(0)
    for hole in (0, 1, 3):
        table = p.table.clone()
        table[0, hole] = -1 if hole != 1 else p.cache.pages
        out = q2d.q2d_attention_cached(q, p.cache, table.cuda(), p.lens().cuda())
        keep = torch.ones(200, dtype=torch.bool)
        keep[64 * hole:64 * hole + 64] = False
        want, _ = ref.attention(q[None], k[None][:, keep], v[None][:, keep], causal=False)
        bound = (2 * U + A) * ref.attention(q[None], k[None][:, keep], v[None][:, keep].abs(), causal=False)[0]
        good = bool(((out.cpu().double() - want[0]).abs() <= bound[0]).all())
        assert good, hole
    none = q2d.q2d_attention_cached(q, p.cache, torch.full_like(p.table, -1).cuda(), p.lens().cuda())
    assert not none.any()
    # a sequence of no tokens, and queries before its first position
    assert not q2d.q2d_attention_cached(q, p.cache, p.table.cuda(), torch.zeros(1, dtype=torch.int32).cuda()).any()
    q3 = q.expand(3, 2, 64).contiguous()
    out = q2d.q2d_attention_cached(q3, p.cache, p.table.cuda(), torch.tensor([2], dtype=torch.int32).cuda())
    assert not out[0].any() and out[1].any() and out[2].any()


@pytest.mark.gpu
def test_decode_step_in_a_graph(q2d):
    """Write and attend captured once and replayed with new tokens and lengths, on a stream of
    its own, beside the same calls made eagerly."""
    counts = [60, 31, 1]
    p, e = (filled(q2d, counts, 2, 128, seed=10) for _ in range(2))
    table = p.table.cuda()
    lens = p.lens().cuda()
    k, v = tokens(3, 2, 128, seed=11)
    q = torch.randn((3, 8, 128), generator=torch.Generator().manual_seed(12)).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)

    def step():
        q2d.q2d_kv_write(p.cache, k, v, table, lens)
        q2d.q2d_attention_cached(q, p.cache, table, lens, out=out)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lens += 1
        step()                                  # the workspace's allocation, outside the capture
    s.synchronize()
    q2d.q2d_kv_write(e.cache, k, v, table, lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        lens += 1
        step()
    for i in range(5):
        nk, nv = tokens(3, 2, 128, seed=20 + i, spread=2.0 ** i)
        k.copy_(nk)
        v.copy_(nv)
        graph.replay()
        torch.cuda.synchronize()
        q2d.q2d_kv_write(e.cache, nk, nv, table, lens)
        want = q2d.q2d_attention_cached(q, e.cache, table, lens)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for n in ("k_codes", "v_codes_t", "k_scales", "v_scales"):
            assert torch.equal(getattr(p.cache, n), getattr(e.cache, n))


@pytest.mark.gpu
def test_refusals(q2d):
    p = filled(q2d, [40, 40], 2, 64)
    k, v = tokens(2, 2, 64)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    table, lens = p.table.cuda(), p.lens().cuda()
    off = torch.tensor([0, 1, 2]).cuda()
    W, R, C = q2d.q2d_kv_write, q2d.q2d_kv_read, q2d.q2d_attention_cached
    bad = [
        lambda: q2d.KVCache(0, 2, 64),
        lambda: q2d.KVCache(4, 2, 64, page_size=48),
        lambda: q2d.KVCache(4, 2, 72),
        lambda: q2d.KVCache(4, 2, 144),
        lambda: W(p.cache, k, v[:1], table, lens),
        lambda: W(p.cache, k.half(), v.half(), table, lens),
        lambda: W(p.cache, k[:, :1], v[:, :1], table, lens),
        lambda: W(p.cache, k, v, table.long(), lens),
        lambda: W(p.cache, k, v, table, lens.long()),
        lambda: W(p.cache, k, v, table, lens, offsets=off[:2]),
        lambda: W(p.cache, k, v, table, lens, offsets=off.int()),
        lambda: W(p.cache, torch.cat((k, k))[:3], torch.cat((v, v))[:3], table, lens),   # 3 rows, 2 sequences
        lambda: W(p.cache, k.cpu(), v.cpu(), table, lens),
        lambda: W(p.cache, k, v, table.cpu(), lens),
        lambda: R(p.cache, table, lens, 2, out_dtype=torch.float16),
        lambda: C(q.float(), p.cache, table, lens),
        lambda: C(q[:, :3], p.cache, table, lens),
        lambda: C(q[:, :, :32], p.cache, table, lens),
        lambda: C(q, p.cache, table, lens, scale=-1.0),
        lambda: C(q, p.cache, table, lens, softcap=math.inf),
        lambda: C(q, p.cache, table, lens, window=-2),
        lambda: C(q, p.cache, table, lens, slopes=torch.zeros(5, device="cuda")),
        lambda: C(q, p.cache, table, lens, out=torch.zeros_like(q)[:1]),
        lambda: C(q, None, table, lens),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(q2d.Q2DError):
            f()
            raise AssertionError("call %d was accepted" % i)
    # no tokens: nothing to do
    assert C(q[:0], p.cache, table, lens).shape == (0, 4, 64)
    W(p.cache, k[:0], v[:0], table, lens)
