"""Numbers that the kernels cannot hold are refused (host only: no call reaches a launch)."""
import ctypes

import pytest

from test_attention_abi import FAKE, cache_of, problem, q2d  # noqa: F401  (q2d: the fixture)

# scale and softcap enter as scale / softcap and 8 / (softcap or scale): float32 numbers each
BAD = [dict(scale=2.0 ** -61), dict(scale=1e-39), dict(scale=2.0 ** 61), dict(scale=3e38), dict(softcap=2.0 ** -61),
       dict(softcap=1e-40), dict(softcap=2.0 ** 61), dict(softcap=3e38)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_scale_and_cap(q2d, bad):
    from paper_2607_24953_amd import attention as A
    a = problem(q2d, **bad)
    assert q2d._lib.q2d_attention_fwd(ctypes.byref(a), None, 0, None) == 2
    assert q2d._lib.q2d_attention_workspace(ctypes.byref(a), 1) == -1
    c, s = cache_of(q2d)
    args = dict(dtype=1, heads_q=8, scale=0.1, q=FAKE, q_stride_token=512, q_stride_head=64, out=FAKE, out_stride_token=512,
                out_stride_head=64)
    g = A._CachedAttention(**dict(args, **bad))
    assert q2d._lib.q2d_attention_cached(ctypes.byref(c), ctypes.byref(s), ctypes.byref(g), FAKE, 1 << 40, None) == 2


def test_ends_of_the_range(q2d):
    for ok in (dict(scale=2.0 ** -60), dict(scale=2.0 ** 60), dict(softcap=2.0 ** -60), dict(softcap=2.0 ** 60)):
        assert q2d._lib.q2d_attention_workspace(ctypes.byref(problem(q2d, **ok)), 0) == 0


@pytest.mark.parametrize("page_size,table_pages", [(65536, 2 ** 14 + 1), (65536, 2 ** 15), (64, 2 ** 24 + 1), (1024, 2 ** 22)], ids=str)
def test_tables_of_too_many_tokens(q2d, page_size, table_pages):
    """A sequence's tokens are counted in 32 bits, with sums of two positions among them: its
    table may name 2^30."""
    from paper_2607_24953_amd import attention as A
    c, s = cache_of(q2d, page_size=page_size, table_pages=table_pages, table_stride=table_pages)
    L = q2d._lib
    for f in (L.q2d_kv_write, L.q2d_kv_read):
        assert f(ctypes.byref(c), ctypes.byref(s), 1, FAKE, 128, 64, FAKE + (1 << 20), 128, 64, None) == 2
    a = A._CachedAttention(dtype=1, heads_q=8, scale=0.1, q=FAKE, q_stride_token=512, q_stride_head=64, out=FAKE + (1 << 20),
                           out_stride_token=512, out_stride_head=64)
    assert L.q2d_attention_cached(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), FAKE, 1 << 40, None) == 2
    assert L.q2d_attention_cached_workspace(ctypes.byref(c), ctypes.byref(s), 8) == -1


def test_the_longest_table(q2d):
    c, s = cache_of(q2d, page_size=65536, table_pages=2 ** 14, table_stride=2 ** 14)
    assert q2d._lib.q2d_attention_cached_workspace(ctypes.byref(c), ctypes.byref(s), 8) >= 0
