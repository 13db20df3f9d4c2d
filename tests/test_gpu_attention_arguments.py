"""Masks and lse of another shape with the right number of elements are refused."""
import pytest
import torch

from test_gpu_attention import make, q2d  # noqa: F401  (q2d: the fixture)

pytestmark = pytest.mark.gpu


def test_transposed_arguments(q2d):
    q, k, v, dout = make(2, 32, 32, 4, 2, 64, torch.bfloat16)
    out, lse = q2d.q2d_attention_fwd(q, k, v)
    docs = torch.zeros((2, 32), dtype=torch.int32, device="cuda")
    q2d.q2d_attention_fwd(q, k, v, documents=docs)
    q2d.q2d_attention_fwd(q, k, v, documents=docs.view(-1))
    with pytest.raises(q2d.Q2DError):
        q2d.q2d_attention_fwd(q, k, v, documents=docs.t().contiguous())
    with pytest.raises(q2d.Q2DError):
        q2d.q2d_attention_fwd(q, k, v, documents=docs.view(4, 16))
    with pytest.raises(q2d.Q2DError):
        q2d.q2d_attention_bwd(dout, q, k, v, out, lse.transpose(1, 2).contiguous())
    q2d.q2d_attention_bwd(dout, q, k, v, out, lse)
    q2d.q2d_attention_bwd(dout, q, k, v, out, lse.view(-1))
