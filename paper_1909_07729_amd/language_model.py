"""A small decoder-only language model on the library's operators, trained on packed documents and then served from a paged cache.

    python -m paper_1909_07729_amd.language_model

Training: ``autograd.kcap_attention`` over documents packed one behind the other (rotated queries and keys, shared heads) and
``autograd.kgelu`` in the MLP.  Serving: ``binding.kcap_append`` puts each layer's rotated keys and its values into the pages of a cache,
``binding.kcap_attention_paged`` reads them, a prompt in pieces and then token by token; the cache belongs to the caller.  Products with
weights, norms and the embedding are torch's; with ``Weights8`` the products of serving are ``binding.kq8_linear`` on weights in 8 bits, and
``binding.ksample`` may choose the tokens.  With ``keep=8`` training keeps 8 bits of each value between an MLP's two products and nothing else.  The documents are synthetic: a random phrase of eight tokens repeated, so that a model
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


class _ActivatedLinear(torch.autograd.Function):
    """K-GELU of h and its product with a weight, of whose inputs the backward pass keeps h in 8 bits: the activation's output, which the weight's
    gradient needs, is rebuilt from them."""

    @staticmethod
    def forward(ctx, h, weight, wide):
        y, codes, scales = (binding.kgelu64_keep8 if wide else binding.kgelu_keep8)(h.contiguous())
        ctx.save_for_backward(codes, scales, weight)
        ctx.wide = wide
        return F.linear(y, weight)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dz):
        codes, scales, weight = ctx.saved_tensors
        backward = binding.kgelu64_keep8_backward if ctx.wide else binding.kgelu_keep8_backward
        dh, y = backward((dz @ weight).contiguous(), codes, scales, rebuild=True)
        return dh, dz.t() @ y, None


class Weights8:
    """A model's weights in 8 bits, as ``serve`` takes them: for each product (integers [outer, inner], scales [outer])."""

    def __init__(self, model):
        def in_8_bits(weights):
            return [binding.kq8_rows(w.detach()) for w in weights]
        self.qkv, self.out, self.up, self.down = (in_8_bits(w) for w in (model.qkv, model.out, model.up, model.down))
        self.head = binding.kq8_rows(model.head.detach())


class LanguageModel(torch.nn.Module):
    def __init__(self, vocabulary=64, width=256, layers=2, heads=4, kv_heads=2, dim=64, longest=512, cap=30.0, intervals=32, device="cuda", keep=None):
        super().__init__()
        if keep not in (None, 8):
            raise ValueError("keep must be None or 8")
        self.heads, self.kv_heads, self.dim, self.cap, self.intervals, self.keep = heads, kv_heads, dim, cap, intervals, keep

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
            if self.keep == 8 and torch.is_grad_enabled():
                x = x + _ActivatedLinear.apply(h, down.bfloat16(), self.intervals == 64).float()
            else:
                x = x + F.linear(autograd.kgelu(h, intervals=self.intervals), down.bfloat16()).float()
        return F.linear(F.rms_norm(x, x.shape[-1:]), self.head)

    def _layers8(self, tokens, attend, weights):
        """The same on weights in 8 bits: tokens go to 8 bits where a product takes them."""
        activated = binding.kq8_linear if self.intervals == 32 else binding.kq8_linear64
        x = self.embedding[tokens]
        for i, (qkv, out, up, down) in enumerate(zip(weights.qkv, weights.out, weights.up, weights.down)):
            h = binding.kq8_linear(F.rms_norm(x, x.shape[-1:]), *qkv).unflatten(-1, (-1, self.dim))
            o = attend(i, *h.split((self.heads, self.kv_heads, self.kv_heads), 1))
            x = x + binding.kq8_linear(o.flatten(1), *out, out_dtype=torch.float32)
            h = binding.kq8_linear(F.rms_norm(x, x.shape[-1:]), *up)
            x = x + activated(h, *down, activation="gelu", out_dtype=torch.float32)
        return binding.kq8_linear(F.rms_norm(x, x.shape[-1:]), *weights.head, out_dtype=torch.float32)

    def forward(self, tokens, offsets, positions):
        """Packed documents: tokens and positions [rows], offsets int32 [documents + 1]."""
        cos, sin = self.cos[positions], self.sin[positions]

        def attend(_, q, k, v):
            return autograd.kcap_attention(_rotated(q, cos, sin), _rotated(k, cos, sin), v, offsets, cap=self.cap, intervals=self.intervals)
        return self._layers(tokens, attend)

    @torch.no_grad()
    def serve(self, tokens, cache: PagedCache, offsets=None, longest=None, weights: Weights8 | None = None):
        """New tokens of every sequence of the cache, one each or, with offsets, a piece of its text; grows the cache.  `longest`: tokens of the
        longest piece, where the caller knows it.  `weights`: the model's in 8 bits, to serve with them."""
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
        logits = self._layers(tokens, attend) if weights is None else self._layers8(tokens, attend, weights)
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
def generate(model, prompts, count, piece=24, page=16, weights=None, sample=None, generator=None):
    """Continuation of prompts (a list of token tensors) by `count` tokens; (tokens [prompts, count], logits of each step).  Greedy, or with `sample`,
    the settings of ``binding.ksample`` (``ksample64`` for a model with 64 intervals), from uniform numbers of `generator` (on the GPU).  `weights`: as for
    ``serve``.  A step whose logits hold a NaN raises ValueError."""
    sequences, longest = len(prompts), max(len(p) for p in prompts)
    if any(len(p) == 0 for p in prompts):
        raise ValueError("a prompt without tokens has no logits to continue from")
    if longest + count > model.cos.shape[0]:
        raise ValueError(f"the model has angles for {model.cos.shape[0]} tokens")
    cache = PagedCache(len(model.qkv), sequences, longest + count, model.kv_heads, model.dim, page)
    last = torch.empty((sequences, model.embedding.shape[0]), device="cuda")
    for start in range(0, longest, piece):
        parts = [p[start:start + piece] for p in prompts]
        offsets = torch.tensor([0] + [len(p) for p in parts]).cumsum(0).int().cuda()
        logits = model.serve(torch.cat(parts), cache, offsets, min(piece, longest - start), weights)
        ends = offsets[1:].long() - 1
        done = torch.tensor([len(p) > 0 for p in parts], device="cuda")
        last[done] = logits[ends[done]]
    sampled = binding.ksample if model.intervals == 32 else binding.ksample64
    tokens, seen = [], [last.clone()]
    for _ in range(count):
        if sample is None:
            tokens.append(seen[-1].argmax(-1))
        else:
            tokens.append(sampled(seen[-1], torch.rand(sequences, generator=generator, device="cuda"), **sample))
        seen.append(model.serve(tokens[-1], cache, weights=weights))
    tokens = torch.stack(tokens, 1)
    if sample is not None and (tokens < 0).any():       # which the embedding takes as its last
        raise ValueError("a step's logits hold a NaN: no token was chosen")
    return tokens, torch.stack(seen[:-1], 1)


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=150)
    parser.add_argument("--intervals", type=int, choices=(32, 64), default=32)
    parser.add_argument("--keep", type=int, choices=(8,), help="bits that training keeps of the values between an MLP's products")
    parser.add_argument("--weights", type=int, choices=(8,), help="bits of the weights that the model is served with")
    parser.add_argument("--temperature", type=float, default=0.0, help="0: the likeliest token")
    parser.add_argument("--top-k", type=int, default=0)
    parser.add_argument("--top-p", type=float, default=1.0)
    parser.add_argument("--min-p", type=float, default=0.0)
    args = parser.parse_args(argv)
    torch.manual_seed(0)
    model = LanguageModel(intervals=args.intervals, keep=args.keep)
    losses = train(model, args.steps)
    for i in range(0, args.steps, max(1, args.steps // 10)):
        print(f"step {i:4d}  loss {losses[i]:.3f}", flush=True)
    tokens, offsets, _ = documents(torch.Generator().manual_seed(1), 8, 64, 100)
    prompts = [tokens[a:b] for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())]
    sample = None
    if args.temperature > 0:
        sample = {"temperature": args.temperature, "top_k": args.top_k, "top_p": args.top_p, "min_p": args.min_p}
    made, _ = generate(model, prompts, 12, weights=Weights8(model) if args.weights else None, sample=sample)
    right = total = 0
    for prompt, new in zip(prompts, made):
        want = [prompt[(len(prompt) + i) % PHRASE].item() for i in range(len(new))]
        right += sum(a == b for a, b in zip(new.tolist(), want))
        total += len(want)
    print(f"loss {losses[0]:.3f} -> {sum(losses[-10:]) / len(losses[-10:]):.3f}; {right} of {total} generated tokens continue their phrase")


if __name__ == "__main__":
    main()
