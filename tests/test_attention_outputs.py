"""Outputs whose rows share memory are refused (host only: no call reaches a launch)."""
import ctypes

import pytest

from test_attention_abi import FAKE, cache_of, problem, q2d  # noqa: F401  (q2d: the fixture)

# of a [batch][length][heads] output with 64 dims: strides that pass one by one
SHARED = [dict(stride_length=64, stride_head=64), dict(stride_length=256, stride_head=64),
          dict(stride_length=448, stride_head=64), dict(stride_length=64, stride_head=640),
          dict(stride_batch=512), dict(stride_batch=64 * 8 * 99), dict(stride_batch=64, stride_length=128, stride_head=12800 - 64)]


@pytest.mark.parametrize("strides", SHARED, ids=str)
def test_forward(q2d, strides):
    a = problem(q2d, **{"out__" + n: x for n, x in strides.items()})
    assert q2d._lib.q2d_attention_fwd(ctypes.byref(a), None, 0, None) == 1


@pytest.mark.parametrize("which", [1, 2, 3])
def test_backward(q2d, which):
    from paper_2607_24953_amd import attention as A
    a = problem(q2d, lse=FAKE)
    g = (A._Heads * 4)()
    at = FAKE
    for h, n, heads in zip(g, (100, 100, 130, 130), (8, 8, 2, 2)):
        h.data, h.stride_batch, h.stride_length, h.stride_head = at, n * heads * 64, heads * 64, 64
        at += 1 << 20
    g[which].stride_length = 64
    refs = [ctypes.byref(g, i * ctypes.sizeof(A._Heads)) for i in range(4)]
    assert q2d._lib.q2d_attention_bwd(ctypes.byref(a), *refs, FAKE, 1 << 40, None) == 1


@pytest.mark.parametrize("token,head", [(128, 128), (64, 64), (64, 128), (256, 64 * 3 + 8)])
def test_cached(q2d, token, head):
    from paper_2607_24953_amd import attention as A
    c, s = cache_of(q2d)
    a = A._CachedAttention(dtype=1, heads_q=8, scale=0.1, q=FAKE, q_stride_token=512, q_stride_head=64, out=FAKE + (1 << 20),
                           out_stride_token=token, out_stride_head=head)
    assert q2d._lib.q2d_attention_cached(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), FAKE, 1 << 40, None) == 1


@pytest.mark.parametrize("token,head", [(64, 64), (64, 256), (120, 64)])
def test_read(q2d, token, head):
    c, s = cache_of(q2d)
    for k, v in (((token, head), (128, 64)), ((128, 64), (token, head))):
        assert q2d._lib.q2d_kv_read(ctypes.byref(c), ctypes.byref(s), 1, FAKE, *k, FAKE + (1 << 20), *v, None) == 1
