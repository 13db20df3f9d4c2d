"""dK and dV where the query heads that share a key head are summed in parts, by workgroups of
their own: against the definition in 64 bits, with the tolerances of the other backward tests.
``parts`` is the rule's answer for the shape (the heads then divide unevenly for 7)."""
import ctypes

import pytest
import torch

from test_gpu_attention import check, make, q2d  # noqa: F401  (q2d: the fixture)

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


def parts_of(q2d, q, k, documents):
    """From the workspace: the parts' sums are what a backward call needs beside two numbers a
    query row and the documents' ranges."""
    from paper_2607_24953_amd import attention as A
    B, Lq, Hq, D = q.shape
    Lk, Hkv = k.shape[1], k.shape[2]
    a = A._Attention(dtype=0, causal=1, batch=B, heads_q=Hq, heads_kv=Hkv, dim=D, len_q=Lq, len_k=Lk, scale=1.0,
                     documents=256 if documents else None)
    up = lambda n: (n + 255) // 256 * 256
    rest = q2d._lib.q2d_attention_workspace(ctypes.byref(a), 1) - 2 * up(B * Hq * Lq * 4)
    rest -= up(B * ((Lk + 63) // 64) * 8) if documents else 0
    n = rest // (B * Lk * Hkv * D * 8)
    assert rest == (up(n * B * Lk * Hkv * D * 8) if n else 0)
    return max(n, 1)


def documents_of(B, L):
    """Documents of unequal length, some padding between and behind them."""
    d = torch.full((B, L), -1, dtype=torch.int32)
    for b in range(B):
        for i, (lo, hi) in enumerate(((0, 0.13), (0.13, 0.14), (0.16, 0.62), (0.62, 0.97))):
            d[b, int(lo * L):int(hi * L)] = i + b
    return d


# few workgroups: 32 keys each
@DTYPES
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("shape,parts", [((1, 1100, 1100, 8, 2), 4), ((1, 700, 690, 7, 1), 4), ((2, 600, 333, 10, 2), 2)],
                         ids=str)
def test_few_workgroups(q2d, shape, parts, D, dtype):
    args = make(*shape, D, dtype, seed=21)
    assert parts_of(q2d, args[0], args[1], False) == parts
    check(q2d, *args)


# 256 workgroups and more: 128 keys each, with the wave pair above 64 dims in bfloat16
@DTYPES
@pytest.mark.parametrize("D", [64, 96, 128])
def test_many_workgroups(q2d, D, dtype):
    args = make(1, 600, 4010, 14, 2, D, dtype, seed=22)
    assert parts_of(q2d, args[0], args[1], False) == 4
    check(q2d, *args, softcap=20.0 if D == 128 else 0.0)


@DTYPES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape,parts", [((1, 1100, 1100, 8, 2), 4), ((1, 600, 4010, 14, 2), 4)], ids=str)
def test_documents(q2d, shape, parts, D, dtype):
    args = make(*shape, D, dtype, seed=23)
    assert parts_of(q2d, args[0], args[1], True) == parts
    check(q2d, *args, documents=documents_of(shape[0], shape[2]))


def test_same_results_each_time(q2d):
    q, k, v, dout = make(1, 1100, 1100, 8, 2, 128, torch.bfloat16, seed=24)
    out, lse = q2d.q2d_attention_fwd(q, k, v)
    first = q2d.q2d_attention_bwd(dout, q, k, v, out, lse)
    for _ in range(3):
        for a, b in zip(first, q2d.q2d_attention_bwd(dout, q, k, v, out, lse)):
            assert torch.equal(a, b)
