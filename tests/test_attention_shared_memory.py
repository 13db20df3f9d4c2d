"""Outputs in the memory of inputs that are still read, or of one another, are refused (host only:
no call reaches a launch)."""
import ctypes

import pytest

from test_attention_abi import FAKE, cache_of, problem, q2d  # noqa: F401  (q2d: the fixture)

STEP = 1 << 20


def forward(q2d, out_data, **strides):
    a = problem(q2d, q__data=FAKE, k__data=FAKE + STEP, v__data=FAKE + 2 * STEP, out__data=out_data,
                **{"out__" + n: x for n, x in strides.items()})
    return q2d._lib.q2d_attention_fwd(ctypes.byref(a), None, 0, None)


# (100 queries of 8 heads, 130 keys of 2 heads, 64 dims, bfloat16, two sequences)
K_BYTES = 2 * 130 * 2 * 64 * 2


@pytest.mark.parametrize("data", [FAKE + STEP, FAKE + 2 * STEP, FAKE + STEP + K_BYTES - 128, FAKE + 128, FAKE + 1024, FAKE - 1024],
                         ids=hex)
def test_forward_out(q2d, data):
    """k, v, the last row of k, and q some heads or rows off."""
    if data < FAKE + STEP:
        data += 4 * STEP
        a = problem(q2d, q__data=FAKE + 4 * STEP, k__data=FAKE + STEP, v__data=FAKE + 2 * STEP, out__data=data)
        assert q2d._lib.q2d_attention_fwd(ctypes.byref(a), None, 0, None) == 1
    else:
        assert forward(q2d, data) == 1


def test_forward_out_of_other_strides(q2d):
    assert forward(q2d, FAKE, stride_batch=51200, stride_length=64, stride_head=6400) == 1


def backward(q2d, **data):
    from paper_2607_24953_amd import attention as A
    where = {n: FAKE + i * STEP for i, n in enumerate(("q", "k", "v", "out", "dout", "dq", "dk", "dv"))}
    where.update({n: where[x] if isinstance(x, str) else x for n, x in data.items()})
    a = problem(q2d, lse=FAKE + 9 * STEP, q__data=where["q"], k__data=where["k"], v__data=where["v"], out__data=where["out"])
    g = (A._Heads * 4)()
    for h, n, heads, name in zip(g, (100, 100, 130, 130), (8, 8, 2, 2), ("dout", "dq", "dk", "dv")):
        h.data, h.stride_batch, h.stride_length, h.stride_head = where[name], n * heads * 64, heads * 64, 64
    refs = [ctypes.byref(g, i * ctypes.sizeof(A._Heads)) for i in range(4)]
    return q2d._lib.q2d_attention_bwd(ctypes.byref(a), *refs, FAKE, 1 << 40, None)


@pytest.mark.parametrize("output,other", [("dk", "k"), ("dk", "v"), ("dv", "k"), ("dv", "v"), ("dk", "q"), ("dv", "q"), ("dk", "dout"),
                                          ("dv", "dout"), ("dq", "k"), ("dq", "v"), ("dk", "dq"), ("dv", "dq"), ("dk", "dv")])
def test_backward(q2d, output, other):
    assert backward(q2d, **{output: other}) == 1


@pytest.mark.parametrize("output,other,off", [("dq", "q", 128), ("dq", "dout", 1024), ("dk", "dv", 128 * 129), ("dv", "dk", 256)])
def test_backward_rows_off(q2d, output, other, off):
    base = {"q": 0, "dout": 4, "dk": 6, "dv": 7}[other]
    assert backward(q2d, **{output: FAKE + base * STEP + off}) == 1


def test_cached(q2d):
    from paper_2607_24953_amd import attention as A
    c, s = cache_of(q2d)
    for off, token, head in ((128, 512, 64), (1024, 512, 64), (0, 64, 64 * 6), (-1024, 512, 64)):
        a = A._CachedAttention(dtype=1, heads_q=8, scale=0.1, q=FAKE + STEP, q_stride_token=512, q_stride_head=64,
                               out=FAKE + STEP + off, out_stride_token=token, out_stride_head=head)
        assert q2d._lib.q2d_attention_cached(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), FAKE, 1 << 40, None) == 1


def test_read(q2d):
    c, s = cache_of(q2d)
    for off in (0, 128, 256, -256):
        assert q2d._lib.q2d_kv_read(ctypes.byref(c), ctypes.byref(s), 1, FAKE + STEP, 128, 64, FAKE + STEP + off, 128, 64, None) == 1
