"""The decoder on root-mean-square norms is the composition that its blocks stand for: stream + attention,
stream + feed-forward part, each of the normed stream, in values, gradients and out of the cache."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def compose(model, x, attends):
    """Logits from the embedded tokens, with the residual's additions written out: every norm gets the whole
    stream and no residual."""
    from paper_2607_24953_amd.autograd import rms_norm
    for b, attend in zip(model.blocks, attends):
        q, k, v = b.qkv(x).unflatten(-1, (-1, b.dim)).split((b.heads, b.kv_heads, b.kv_heads), dim=-2)
        x = x + b.o(attend(q, k, v).flatten(-2))
        x = x + b.down(torch.relu(b.up(x)))
    return rms_norm(x, model.norm_weight, y_dtype=torch.float32) @ model.embedding.weight.t()


def calls(model, count=None):
    """The layers' call counters, which pick their random bits."""
    layers = [m for m in model.modules() if hasattr(m, "_calls")]
    if count is not None:
        for m, c in zip(layers, count):
            m._calls = c
    return [m._calls for m in layers]


@pytest.fixture
def model():
    from paper_2607_24953_amd.decoder import Decoder
    torch.manual_seed(3)
    m = Decoder(norm="rms", layers=3)
    with torch.no_grad():
        for b in m.blocks:
            for p in (b.qkv.norm_weight, b.up.norm_weight):
                p += 0.2 * torch.randn_like(p)
        m.norm_weight += 0.2 * torch.randn_like(m.norm_weight)
    return m


@pytest.mark.parametrize("shape", [(2, 65), (1, 1), (3, 128)], ids=str)
def test_training_path(model, shape):
    from paper_2607_24953_amd.autograd import attention
    tokens = torch.randint(64, shape, device=DEV, generator=torch.Generator(DEV).manual_seed(4))
    documents = (torch.arange(shape[1], device=DEV, dtype=torch.int32) // 40).expand(shape).contiguous()
    dlogits = torch.randn((*shape, 64), device=DEV, generator=torch.Generator(DEV).manual_seed(5))
    start, got = calls(model), []
    attends = [lambda q, k, v, b=b: attention(q, k, v, softcap=b.softcap, slopes=model.slopes, documents=documents)
               for b in model.blocks]
    for run in (lambda: model(tokens, documents), lambda: compose(model, model.embedding(tokens), attends)):
        calls(model, start)
        model.zero_grad(set_to_none=True)
        logits = run()
        logits.backward(dlogits)
        got.append((logits.detach(), {k: p.grad for k, p in model.named_parameters()}))
    (a, ga), (b, gb) = got
    # the additions are the same ones, in float32
    assert torch.equal(a, b)
    for k in ga:
        if k == "embedding.weight":
            # (torch sums over equal tokens in an order of its own; float32)
            assert float((ga[k] - gb[k]).norm() / gb[k].norm()) <= 1e-5
        else:
            assert torch.equal(ga[k], gb[k]), k


def test_cached_path(model):
    from paper_2607_24953_amd import q2d_attention_cached, q2d_kv_write
    tokens = torch.randint(64, (2, 9), device=DEV, generator=torch.Generator(DEV).manual_seed(6))
    table = torch.arange(4, dtype=torch.int32, device=DEV).view(2, 2)
    two = [model.caches(4), model.caches(4)]
    # a prompt of six tokens, then one token at a time
    for first, last in ((0, 6), (6, 7), (7, 8), (8, 9)):
        new, lens = tokens[:, first:last].reshape(-1), torch.full((2,), last, dtype=torch.int32, device=DEV)

        def attend(cache, b):
            def f(q, k, v):
                q2d_kv_write(cache, k, v, table, lens, None)
                return q2d_attention_cached(q, cache, table, lens, None, softcap=b.softcap, slopes=model.slopes)
            return f
        with torch.no_grad():
            got = model.step(new, two[0], table, lens)
            want = compose(model, model.embedding(new), [attend(c, b) for c, b in zip(two[1], model.blocks)])
        assert got.shape == (new.numel(), 64) and torch.equal(got, want), (first, last)
