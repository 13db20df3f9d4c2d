"""Host-side checks of the attention and cache entry points (no GPU, no kernel is launched):
sizes, workspaces and the status of every refused argument."""
import ctypes

import pytest

FAKE = 0x1000


@pytest.fixture(scope="module")
def q2d():
    import paper_2607_24953_amd as q
    return q


def problem(q2d, **kw):
    from paper_2607_24953_amd import attention as A
    a = A._Attention(dtype=1, causal=1, batch=2, heads_q=8, heads_kv=2, dim=64, len_q=100, len_k=130, window=0,
                     scale=0.125, softcap=0.0)
    for h, n, heads in ((a.q, 100, 8), (a.k, 130, 2), (a.v, 130, 2), (a.out, 100, 8)):
        h.data, h.stride_batch, h.stride_length, h.stride_head = FAKE, n * heads * 64, heads * 64, 64
    for k, v in kw.items():
        at = a
        *path, last = k.split("__")
        for name in path:
            at = getattr(at, name)
        setattr(at, last, v)
    return a


def fwd(q2d, a, ws=None, size=0):
    return q2d._lib.q2d_attention_fwd(ctypes.byref(a), ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=2), 1), (dict(causal=2), 1), (dict(batch=0), 1), (dict(heads_q=7), 1), (dict(heads_kv=0), 1),
    (dict(len_q=0), 1), (dict(len_k=-1), 1), (dict(window=-1), 1), (dict(scale=0.0), 1), (dict(scale=float("inf")), 1),
    (dict(scale=float("nan")), 1), (dict(softcap=-1.0), 1), (dict(softcap=float("nan")), 1), (dict(dim=0), 1),
    (dict(dim=60), 2), (dict(dim=136), 2), (dict(len_k=2 ** 30 + 1), 2), (dict(batch=2 ** 31 - 1, len_k=2 ** 30), 2),
    (dict(q__data=None), 1), (dict(k__data=FAKE + 8), 1), (dict(v__stride_length=132), 1), (dict(q__stride_head=-64), 1),
    (dict(out__stride_head=0), 1), (dict(out__stride_length=32), 1), (dict(k__stride_length=2 ** 22), 2),
    (dict(k__stride_batch=2 ** 46), 0x2), (dict(slopes=FAKE + 2), 1), (dict(documents=FAKE), 1), (dict(lse=FAKE + 1), 1),
], ids=str)
def test_forward_refusals(q2d, bad, status):
    if "k__stride_batch" in bad:
        bad = dict(bad, batch=4)                  # the last element lies beyond 2^47
    assert fwd(q2d, problem(q2d, **bad)) == status


def test_forward_null():
    import paper_2607_24953_amd as q
    assert q._lib.q2d_attention_fwd(None, None, 0, None) == 1
    assert q._lib.q2d_attention_workspace(None, 0) == -1


def test_workspaces(q2d):
    W = lambda back, **kw: q2d._lib.q2d_attention_workspace(ctypes.byref(problem(q2d, **kw)), back)
    assert W(0) == 0 and W(0, documents=FAKE) == 256
    assert W(2) == -1 and W(0, dim=60) == -1
    # two rows of float32 a query row, 256-byte steps; parts only with shared key heads
    rows = (2 * 8 * 100 * 4 + 255) // 256 * 256
    assert W(1, heads_kv=8) == 2 * rows
    assert W(1, heads_kv=8, documents=FAKE) == 2 * rows + 256
    a = problem(q2d, documents=FAKE)
    assert fwd(q2d, a, None, 0) == 1 and fwd(q2d, a, FAKE + 16, 256) == 1 and fwd(q2d, a, FAKE, 255) == 1


def test_backward_refusals(q2d):
    from paper_2607_24953_amd import attention as A
    a = problem(q2d, lse=FAKE)
    g = (A._Heads * 4)()
    for h, n, heads in zip(g, (100, 100, 130, 130), (8, 8, 2, 2)):
        h.data, h.stride_batch, h.stride_length, h.stride_head = FAKE, n * heads * 64, heads * 64, 64
    size = q2d._lib.q2d_attention_workspace(ctypes.byref(a), 1)
    refs = [ctypes.byref(g, i * ctypes.sizeof(A._Heads)) for i in range(4)]
    B = lambda a, refs, ws=FAKE, n=size: q2d._lib.q2d_attention_bwd(ctypes.byref(a), *refs, ws, n, None)
    assert B(a, refs, None) == 1 and B(a, refs, FAKE, size - 1) == 1
    assert B(problem(q2d), refs) == 1                                  # no lse
    for i in range(4):
        assert B(a, refs[:i] + [None] + refs[i + 1:]) == 1
    g[2].stride_head = 0                                               # an output whose rows share memory
    assert B(a, refs) == 1


def cache_of(q2d, **kw):
    from paper_2607_24953_amd import attention as A
    c = A._Cache(pages=10, heads=2, dim=64, page_size=64, k_codes=FAKE, v_codes_t=FAKE, k_scales=FAKE, v_scales=FAKE)
    s = A._Sequences(batch=3, table_pages=4, tokens=6, table_stride=4, offsets=FAKE, lens=FAKE, table=FAKE)
    for k, v in kw.items():
        setattr(c if hasattr(c, k) else s, k, v)
    return c, s


CACHE_BAD = [(dict(pages=0), 1), (dict(heads=-1), 1), (dict(page_size=48), 1), (dict(dim=72), 2), (dict(dim=144), 2),
             (dict(page_size=65568), 2), (dict(pages=2 ** 30), 2), (dict(k_codes=None), 1), (dict(v_codes_t=FAKE + 4), 1),
             (dict(k_scales=None), 1), (dict(batch=0), 1), (dict(tokens=-1), 1), (dict(table_pages=0), 1),
             (dict(table_stride=3), 1), (dict(lens=None), 1), (dict(table=None), 1), (dict(table=FAKE + 2), 1),
             (dict(offsets=FAKE + 4), 1), (dict(offsets=None, tokens=7), 1), (dict(batch=2 ** 20 + 1), 2)]


@pytest.mark.parametrize("bad,status", CACHE_BAD, ids=str)
def test_cache_refusals(q2d, bad, status):
    from paper_2607_24953_amd import attention as A
    L = q2d._lib
    c, s = cache_of(q2d, **bad)
    for f in (L.q2d_kv_write, L.q2d_kv_read):
        assert f(ctypes.byref(c), ctypes.byref(s), 1, FAKE, 128, 64, FAKE, 128, 64, None) == status
    a = A._CachedAttention(dtype=1, heads_q=8, scale=0.1, q=FAKE, q_stride_token=512, q_stride_head=64, out=FAKE,
                           out_stride_token=512, out_stride_head=64)
    assert L.q2d_attention_cached(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), FAKE, 1 << 30, None) == status


def test_cached_attention_refusals(q2d):
    from paper_2607_24953_amd import attention as A
    L = q2d._lib
    c, s = cache_of(q2d)

    def call(ws=FAKE, n=1 << 30, **kw):
        a = A._CachedAttention(dtype=1, heads_q=8, scale=0.1, q=FAKE, q_stride_token=512, q_stride_head=64, out=FAKE,
                               out_stride_token=512, out_stride_head=64)
        for k, v in kw.items():
            setattr(a, k, v)
        return L.q2d_attention_cached(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), ws, n, None)

    for bad, status in ((dict(dtype=0), 2), (dict(dtype=3), 1), (dict(heads_q=3), 1), (dict(heads_q=0), 1),
                        (dict(scale=0.0), 1), (dict(softcap=-1.0), 1), (dict(window=-1), 1), (dict(slopes=FAKE + 1), 1),
                        (dict(prefix=FAKE + 2), 1), (dict(q=None), 1), (dict(q_stride_token=100), 1),
                        (dict(out_stride_head=32), 1), (dict(q=FAKE + 8), 1), (dict(heads_q=2 ** 30), 2)):
        assert call(**bad) == status, bad
    assert L.q2d_attention_cached(ctypes.byref(c), ctypes.byref(s), None, None, 0, None) == 1
    c, s = cache_of(q2d, table_pages=100, table_stride=100)
    need = L.q2d_attention_cached_workspace(ctypes.byref(c), ctypes.byref(s), 8)
    assert need > 0 and call(None, need) == 1 and call(FAKE, need - 1) == 1 and call(FAKE + 16, need) == 1
    assert L.q2d_attention_cached_workspace(ctypes.byref(c), ctypes.byref(s), 7) == -1
    assert L.q2d_attention_cached_workspace(None, ctypes.byref(s), 8) == -1


def test_cache_layout(q2d):
    from paper_2607_24953_amd import attention as A
    c, sizes = A._Cache(), (ctypes.c_int64 * 4)()
    assert q2d._lib.q2d_kv_cache_init(ctypes.byref(c), 5, 3, 80, 96, sizes) == 0
    assert list(sizes) == [5 * 3 * 96 * 80, 5 * 3 * 96 * 80, 45, 45] and c.k_codes is None and c.page_size == 96
    assert q2d._lib.q2d_kv_cache_init(None, 5, 3, 80, 96, sizes) == 1
    t = q2d.KVCache(5, 3, 80, page_size=96, device="cpu")
    assert t.k_codes.shape == (5, 3, 96, 80) and t.v_codes_t.shape == (5, 3, 3, 80, 32) and t.k_scales.shape == (5, 3, 3)


def test_binding_refuses_host_tensors(q2d):
    import torch
    x = torch.zeros((1, 8, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(q2d.Q2DError):
        q2d.q2d_attention_fwd(x, x, x)
    c = q2d.KVCache(2, 2, 64, device="cpu")
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    with pytest.raises(q2d.Q2DError):
        q2d.q2d_kv_write(c, x[0, :1], x[0, :1], table, lens)
    with pytest.raises(q2d.Q2DError):
        q2d.q2d_attention_cached(x[0, :1], c, table, lens)
