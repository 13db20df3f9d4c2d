"""A small decoder on the library's operators: quantized linear layers with attention between
them, trained on packed documents and then answering from a paged 8-bit key/value cache.

``Decoder.forward`` is the training path (Q2DLinear, ``autograd.attention`` with a document
mask); ``Decoder.step`` takes new tokens of several sequences, prompts or single tokens,
through q2d_kv_write and q2d_attention_cached.  Norms are torch's LayerNorm, or with
``norm="rms"`` the library's root-mean-square norm, which adds the residual and writes the
operands of the linear layer behind it (Q2DNormLinear).  ``train`` clips the gradients by their
global norm where asked to (q2d_clip_grads).

``python -m paper_2607_24953_amd.decoder`` trains one on documents that repeat a random phrase and
prints the loss and how well it continues such documents out of the cache.
"""
from __future__ import annotations

import argparse
import sys

import torch

from . import KVCache, q2d_attention_cached, q2d_clip_grads, q2d_kv_write
from .autograd import Q2DLinear, Q2DNormLinear, attention, rms_norm


class Block(torch.nn.Module):
    """Attention and a two-layer feed-forward part, each on the normed residual stream."""

    Normed = Q2DLinear      # the layers behind a norm

    def __init__(self, hidden, heads, kv_heads, softcap, device):
        super().__init__()
        self.heads, self.kv_heads, self.dim, self.softcap = heads, kv_heads, hidden // heads, softcap
        self.qkv = self.Normed(hidden, (heads + 2 * kv_heads) * self.dim, device=device)
        self.o = Q2DLinear(hidden, hidden, device=device)
        self.up = self.Normed(hidden, 4 * hidden, device=device)
        self.down = Q2DLinear(4 * hidden, hidden, device=device)
        if self.Normed is Q2DLinear:
            self.norms = torch.nn.ModuleList(torch.nn.LayerNorm(hidden, device=device) for _ in range(2))

    def forward(self, x, attend):
        """attend(q, k, v) -> attention's output, all [..., heads, dim]"""
        dt = torch.bfloat16
        y = self.qkv(self.norms[0](x).to(dt)).unflatten(-1, (-1, self.dim))
        q, k, v = y.split((self.heads, self.kv_heads, self.kv_heads), dim=-2)
        x = x + self.o(attend(q, k, v).flatten(-2)).float()
        return x + self.down(torch.relu(self.up(self.norms[1](x).to(dt)))).float()


class RMSBlock(Block):
    """The same on root-mean-square norms: each adds the branch before it to the stream and writes
    the operands of the linear layer behind it."""

    Normed = Q2DNormLinear

    def forward(self, x, attend, branch=None):
        """The stream x and what is still to be added to it (None: nothing) -> the same behind this
        block."""
        if branch is None:
            y = self.qkv(x)
        else:
            y, x = self.qkv(x, branch)
        q, k, v = y.unflatten(-1, (-1, self.dim)).split((self.heads, self.kv_heads, self.kv_heads), dim=-2)
        y, x = self.up(x, self.o(attend(q, k, v).flatten(-2)))
        return x, self.down(torch.relu(y))


class Decoder(torch.nn.Module):
    """Token embedding, blocks, and logits by the embedding.  Positions enter by the heads'
    distance bias (slopes), which training and the cached path share."""

    def __init__(self, vocabulary=64, hidden=256, layers=2, heads=4, kv_heads=2, softcap=30.0, device="cuda",
                 norm="layer"):
        super().__init__()
        if norm not in ("layer", "rms"):
            raise ValueError("norm must be 'layer' or 'rms'")
        self.embedding = torch.nn.Embedding(vocabulary, hidden, device=device)
        torch.nn.init.normal_(self.embedding.weight, std=hidden ** -0.5)
        self.rms = norm == "rms"
        block = RMSBlock if self.rms else Block
        self.blocks = torch.nn.ModuleList(block(hidden, heads, kv_heads, softcap, device) for _ in range(layers))
        if self.rms:
            self.norm_weight = torch.nn.Parameter(torch.ones(hidden, device=device))
        else:
            self.norm = torch.nn.LayerNorm(hidden, device=device)
        # half the heads look near, half far
        slopes = [2.0 ** -(1 + 7 * i / max(1, heads - 1)) for i in range(heads)]
        self.register_buffer("slopes", torch.tensor(slopes, dtype=torch.float32, device=device))

    def _block(self, b, x, branch, attend):
        return b(x, attend, branch) if self.rms else (b(x, attend), None)

    def _logits(self, x, branch):
        if self.rms:
            y = rms_norm(x, self.norm_weight, residual=branch, y_dtype=torch.float32)
            y = y if branch is None else y[0]
        else:
            y = self.norm(x)
        return y @ self.embedding.weight.t()

    def forward(self, tokens, documents=None):
        """Logits of tokens [batch, length]; documents [batch, length] (int32): packed rows."""
        x, branch = self.embedding(tokens), None
        for b in self.blocks:
            def attend(q, k, v):
                return attention(q, k, v, softcap=b.softcap, slopes=self.slopes, documents=documents)
            x, branch = self._block(b, x, branch, attend)
        return self._logits(x, branch)

    def caches(self, pages, page_size=64):
        b = self.blocks[0]
        return [KVCache(pages, b.kv_heads, b.dim, page_size=page_size, device=self.slopes.device) for _ in self.blocks]

    @torch.no_grad()
    def step(self, tokens, caches, table, lens, offsets=None):
        """Logits of the new tokens [tokens] of several sequences (rows offsets[b] ..
        offsets[b + 1]; None: equally many each), which join the caches; lens counts them."""
        x, branch = self.embedding(tokens), None
        for b, cache in zip(self.blocks, caches):
            def attend(q, k, v):
                q2d_kv_write(cache, k, v, table, lens, offsets)
                return q2d_attention_cached(q, cache, table, lens, offsets, softcap=b.softcap, slopes=self.slopes)
            x, branch = self._block(b, x, branch, attend)
        return self._logits(x, branch)

    @torch.no_grad()
    def generate(self, prompts, count, page_size=64):
        """Greedy continuations [len(prompts), count] of a list of prompts (1-D token tensors, none
        of them empty: there is nothing to continue)."""
        device = self.slopes.device
        n = [len(p) for p in prompts]
        if not n or min(n) == 0 or count < 0:
            raise ValueError("prompts of one token or more, and a count of 0 or more, are expected")
        if count == 0:
            return torch.empty((len(n), 0), dtype=torch.int64, device=device)
        per = -(-(max(n) + count) // page_size)
        caches = self.caches(len(n) * per, page_size)
        table = torch.arange(len(n) * per, dtype=torch.int32, device=device).view(len(n), per)
        lens = torch.tensor(n, dtype=torch.int32, device=device)
        ends = torch.tensor(n, device=device).cumsum(0)
        offsets = torch.cat((ends.new_zeros(1), ends))
        logits = self.step(torch.cat([p.to(device) for p in prompts]), caches, table, lens, offsets)[ends - 1]
        out = [logits.argmax(-1)]
        for _ in range(count - 1):
            lens = lens + 1
            out.append(self.step(out[-1], caches, table, lens).argmax(-1))
        return torch.stack(out, 1)


def repeated_phrases(rows, length, vocabulary, generator, device):
    """Rows of packed documents, each a random phrase over and over; tokens, documents and where
    the next token follows from the document (its second repetition on)."""
    tokens = torch.zeros((rows, length + 1), dtype=torch.int64)
    documents = torch.zeros((rows, length), dtype=torch.int32)
    known = torch.zeros((rows, length), dtype=torch.bool)
    for r in range(rows):
        at, doc = 0, 0
        while at < length:
            n = int(torch.randint(4, 13, (1,), generator=generator))
            size = min(n * int(torch.randint(3, 9, (1,), generator=generator)), length + 1 - at)
            phrase = torch.randint(vocabulary, (n,), generator=generator)
            tokens[r, at:at + size] = phrase.repeat(-(-size // n))[:size]
            documents[r, at:at + size] = doc
            known[r, at + n - 1:at + size - 1] = True
            at, doc = at + size, doc + 1
    return tokens.to(device), documents.to(device), known.to(device)


def train(model, steps, rows=16, length=256, vocabulary=64, lr=1e-3, seed=0, clip=None):
    """Trains on repeated_phrases; returns the loss of every step.  clip: the largest global norm
    of the gradients."""
    g = torch.Generator().manual_seed(seed)
    opt = torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.0)
    losses = []
    for i in range(steps):
        tokens, documents, known = repeated_phrases(rows, length, vocabulary, g, model.slopes.device)
        for group in opt.param_groups:
            group["lr"] = lr * min(1.0, (i + 1) / 50)
        logits = model(tokens[:, :-1], documents)
        loss = torch.nn.functional.cross_entropy(logits[known], tokens[:, 1:][known])
        opt.zero_grad(set_to_none=True)
        loss.backward()
        if clip is not None:
            q2d_clip_grads([p.grad for p in model.parameters() if p.grad is not None], clip)
        opt.step()
        losses.append(float(loss.detach()))
    return losses


def main(argv=None) -> int:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--norm", choices=["layer", "rms"], default="layer")
    p.add_argument("--clip", type=float, default=None, help="largest global norm of the gradients")
    a = p.parse_args(argv)
    torch.manual_seed(0)
    model = Decoder(norm=a.norm)
    losses = train(model, a.steps, clip=a.clip)
    for i in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d  loss %.3f" % (i, losses[i]), flush=True)
    g = torch.Generator().manual_seed(1)
    phrases = [torch.randint(64, (int(n),), generator=g) for n in torch.randint(4, 13, (16,), generator=g)]
    prompts = [f.repeat(3) for f in phrases]
    got = model.generate(prompts, 24).cpu()
    want = torch.stack([f.repeat(8)[:24] for f in phrases])
    print("continued from the cache: %.1f %% of 24 tokens right" % (100 * float((got == want).float().mean())))
    return 0


if __name__ == "__main__":
    sys.exit(main())
