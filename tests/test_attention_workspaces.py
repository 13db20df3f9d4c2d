"""Workspace of backward calls whose key heads are summed in parts (host only)."""
import ctypes

import pytest


def up(n):
    return (n + 255) // 256 * 256


@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,D,documents,parts", [
    (1, 1100, 1100, 8, 2, 64, False, 4), (1, 700, 690, 7, 1, 72, False, 4), (2, 600, 333, 10, 2, 128, False, 2),
    (1, 600, 4010, 14, 2, 96, False, 4), (1, 16384, 16384, 32, 8, 64, True, 4), (1, 1100, 1100, 8, 8, 64, True, 1),
    (4, 1024, 1024, 32, 8, 128, False, 1),
])
def test_parts(B, Lq, Lk, Hq, Hkv, D, documents, parts):
    import paper_2607_24953_amd as q2d
    from paper_2607_24953_amd import attention as A
    a = A._Attention(dtype=1, causal=1, batch=B, heads_q=Hq, heads_kv=Hkv, dim=D, len_q=Lq, len_k=Lk, scale=1.0,
                     documents=256 if documents else None)
    # lse and delta of the query rows, a float32 dK and dV a part, the documents' ranges
    want = 2 * up(B * Hq * Lq * 4) + (up(parts * B * Lk * Hkv * D * 8) if parts > 1 else 0)
    want += up(B * ((Lk + 63) // 64) * 8) if documents else 0
    assert q2d._lib.q2d_attention_workspace(ctypes.byref(a), 1) == want
