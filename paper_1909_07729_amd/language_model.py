"""A small decoder-only language model on the library's operators, trained on packed documents and then served from a paged cache.

    python -m paper_1909_07729_amd.language_model

Training: ``autograd.kcap_attention`` over documents packed one behind the other (rotated queries and keys, shared heads) and
``autograd.kgelu`` in the MLP.  Serving: ``binding.kcap_append`` puts each layer's rotated keys and its values into the pages of a cache,
``binding.kcap_attention_paged`` reads them, a prompt in pieces and then token by token; the cache belongs to the caller.  Products with
weights, norms and the embedding are torch's.  The documents are synthetic: a random phrase of eight tokens repeated, so that a model
that attends to what it has read predicts all but the first round.
"""
from __future__ import annotations

import argparse
import math

import torch
import torch.nn.functional as F

from . import autograd, binding


def angles(positions: int, dim: int, device="cuda"):
    """(cos, sin) [positions, dim / 2] Float32, formed in 64 bits."""
    turn = torch.outer(torch.arange(positions, dtype=torch.float64), 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim))
    return turn.cos().float().to(device), turn.sin().float().to(device)


def _rotated(x, cos, sin):
    """The rotation of ``kcap_append`` (pairs x_i, x_{i + dim/2}) where a gradient is wanted; x [rows, heads, dim]."""
    a, b = x.float().chunk(2, -1)
    cos, sin = cos[:, None, :], sin[:, None, :]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)


class PagedCache:
    """Keys and values of every layer in pages.  Each sequence has pages of its own for `longest` tokens, handed out at the start in a random
    order, so that no sequence's pages are neighbours.  ``held``, counted on the host: keys that the longest sequence has at most."""

    def __init__(self, layers, sequences, longest, kv_heads, dim, page=16, device="cuda"):
        most = -(-longest // page)
        shape = (sequences * most, page, kv_heads, dim)
        self.k, self.v = ([torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(layers)] for _ in range(2))
        order = torch.randperm(sequences * most, generator=torch.Generator().manual_seed(0))
        self.pages = order.view(sequences, most).int().to(device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.page, self.held = page, 0


class LanguageModel(torch.nn.Module):
    def __init__(self, vocabulary=64, width=256, layers=2, heads=4, kv_heads=2, dim=64, longest=512, cap=30.0, intervals=32, device="cuda"):
        super().__init__()
        self.heads, self.kv_heads, self.dim, self.cap, self.intervals = heads, kv_heads, dim, cap, intervals

        def weights(*shape):
            return torch.nn.Parameter(torch.randn(*shape, device=device) / math.sqrt(shape[-1]))
        self.embedding = torch.nn.Parameter(torch.randn(vocabulary, width, device=device))
        self.head = weights(vocabulary, width)
        self.qkv = torch.nn.ParameterList(weights((heads + 2 * kv_heads) * dim, width) for _ in range(layers))
        self.out = torch.nn.ParameterList(weights(width, heads * dim) for _ in range(layers))
        self.up = torch.nn.ParameterList(weights(4 * width, width) for _ in range(layers))
        self.down = torch.nn.ParameterList(weights(width, 4 * width) for _ in range(layers))
        cos, sin = angles(longest, dim, device)
        self.register_buffer("cos", cos)
        self.register_buffer("sin", sin)

    def _layers(self, tokens, attend):
        """Logits [tokens, vocabulary]; ``attend(layer, q, k, v)`` from and to [tokens, heads, dim]."""
        x = self.embedding[tokens]
        for i, (qkv, out, up, down) in enumerate(zip(self.qkv, self.out, self.up, self.down)):
            h = F.linear(F.rms_norm(x, x.shape[-1:]).bfloat16(), qkv.bfloat16()).unflatten(-1, (-1, self.dim))
            o = attend(i, *h.split((self.heads, self.kv_heads, self.kv_heads), 1))
            x = x + F.linear(o.flatten(1), out.bfloat16()).float()
            h = F.linear(F.rms_norm(x, x.shape[-1:]).bfloat16(), up.bfloat16())
            x = x + F.linear(autograd.kgelu(h, intervals=self.intervals), down.bfloat16()).float()
        return F.linear(F.rms_norm(x, x.shape[-1:]), self.head)

    def forward(self, tokens, offsets, positions):
        """Packed documents: tokens and positions [rows], offsets int32 [documents + 1]."""
        cos, sin = self.cos[positions], self.sin[positions]

        def attend(_, q, k, v):
            return autograd.kcap_attention(_rotated(q, cos, sin), _rotated(k, cos, sin), v, offsets, cap=self.cap, intervals=self.intervals)
        return self._layers(tokens, attend)

    @torch.no_grad()
    def serve(self, tokens, cache: PagedCache, offsets=None, longest=None):
        """New tokens of every sequence of the cache, one each or, with offsets, a piece of its text; grows the cache.  `longest`: tokens of the
        longest piece, where the caller knows it."""
        room = min(self.cos.shape[0], cache.pages.shape[1] * cache.page)
        if longest is None:
            longest = 1 if offsets is None else min(tokens.shape[0], max(room - cache.held, 0))
        held = cache.held + longest
        if held > room:
            raise ValueError(f"{held} tokens of a sequence are more than the model's angles or the cache's pages hold")
        paged = binding.kcap_attention_paged if self.intervals == 32 else binding.kcap_attention64_paged
        new = torch.ones_like(cache.lengths) if offsets is None else offsets.diff()
        lengths = cache.lengths + new
        pages = cache.pages[:, :-(-held // cache.page)]     # those that the longest sequence needs: the work is cut by them

        def attend(i, q, k, v):
            q = binding.kcap_append(q, k, v, cache.k[i], cache.v[i], pages, cache.lengths, offsets, cos=self.cos, sin=self.sin)
            return paged(q, cache.k[i], cache.v[i], pages, lengths, offsets, cap=self.cap)
        logits = self._layers(tokens, attend)
        cache.lengths, cache.held = lengths, held
        return logits


PHRASE = 8


def documents(generator, count, vocabulary, longest):
    """(tokens, offsets, positions) of documents of 16 to `longest` tokens that repeat a random phrase."""
    texts = []
    for _ in range(count):
        phrase = torch.randint(0, vocabulary, (PHRASE,), generator=generator)
        n = int(torch.randint(2 * PHRASE, longest + 1, (1,), generator=generator))
        texts.append(phrase.repeat(-(-n // PHRASE))[:n])
    offsets = torch.tensor([0] + [len(t) for t in texts]).cumsum(0).int().cuda()
    return torch.cat(texts).cuda(), offsets, torch.cat([torch.arange(len(t)) for t in texts]).cuda()


def train(model, steps, batch=16, longest=128, seed=0):
    """Mean losses of the steps."""
    if longest > model.cos.shape[0]:
        raise ValueError(f"the model has angles for {model.cos.shape[0]} tokens")
    generator = torch.Generator().manual_seed(seed)
    optimizer = torch.optim.Adam(model.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        tokens, offsets, positions = documents(generator, batch, model.embedding.shape[0], longest)
        logits = model(tokens, offsets, positions)
        follows = positions[1:] != 0        # the next row is of the same document
        loss = F.cross_entropy(logits[:-1][follows], tokens[1:][follows])
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


@torch.no_grad()
def generate(model, prompts, count, piece=24, page=16):
    """Greedy continuation of prompts (a list of token tensors) by `count` tokens; (tokens [prompts, count], logits of each step)."""
    sequences, longest = len(prompts), max(len(p) for p in prompts)
    if longest + count > model.cos.shape[0]:
        raise ValueError(f"the model has angles for {model.cos.shape[0]} tokens")
    cache = PagedCache(len(model.qkv), sequences, longest + count, model.kv_heads, model.dim, page)
    last = torch.empty((sequences, model.embedding.shape[0]), device="cuda")
    for start in range(0, longest, piece):
        parts = [p[start:start + piece] for p in prompts]
        offsets = torch.tensor([0] + [len(p) for p in parts]).cumsum(0).int().cuda()
        logits = model.serve(torch.cat(parts), cache, offsets, min(piece, longest - start))
        ends = offsets[1:].long() - 1
        done = torch.tensor([len(p) > 0 for p in parts], device="cuda")
        last[done] = logits[ends[done]]
    tokens, seen = [], [last.clone()]
    for _ in range(count):
        tokens.append(seen[-1].argmax(-1))
        seen.append(model.serve(tokens[-1], cache))
    return torch.stack(tokens, 1), torch.stack(seen[:-1], 1)


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=150)
    parser.add_argument("--intervals", type=int, choices=(32, 64), default=32)
    args = parser.parse_args(argv)
    torch.manual_seed(0)
    model = LanguageModel(intervals=args.intervals)
    losses = train(model, args.steps)
    for i in range(0, args.steps, max(1, args.steps // 10)):
        print(f"step {i:4d}  loss {losses[i]:.3f}", flush=True)
    tokens, offsets, _ = documents(torch.Generator().manual_seed(1), 8, 64, 100)
    prompts = [tokens[a:b] for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())]
    made, _ = generate(model, prompts, 12)
    right = total = 0
    for prompt, new in zip(prompts, made):
        want = [prompt[(len(prompt) + i) % PHRASE].item() for i in range(len(new))]
        right += sum(a == b for a, b in zip(new.tolist(), want))
        total += len(want)
    print(f"loss {losses[0]:.3f} -> {sum(losses[-10:]) / len(losses[-10:]):.3f}; {right} of {total} generated tokens continue their phrase")


if __name__ == "__main__":
    main()
