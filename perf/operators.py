"""Attention whose scores are capped through K-TanH, as cases that can be timed and checked: over packed
documents (inference and training), over a paged cache (single tokens and pieces of prompts), and the
appending of rotated keys and of values to that cache.

A case is a plain dict.  ``listed()`` names a few, ``draw(rng)`` makes more of the same ranges,
``prepare(case, seed)`` builds what a program has in hand before the call, ``run(state)`` is one pass,
``work(case)`` the bytes and operations that the pass cannot do without, ``exact(case, seed)`` the same
outputs in 64 bits.  With ``own`` false ``run`` computes them with elementary torch operations in 32 bits,
with ``own`` true through the library.

The score of a query and a key is  cap * K(scale * (q . k) / cap),  K being K-TanH (arXiv:1909.07729) in its
Float32 form: on each interval of its table K is the line  2^(E-E_i-r) |x| + 2^(E-127) (1 - 2^-r + b/128).
The weights are the softmax of the scores over the keys that the query sees; a query that sees no key has
the output 0 and a log-sum of -infinity.

Kinds of case
  attend   packed documents, output and log-sums (binding): a prompt, or the forward pass of training
  train    output and the gradients of q, k and v (autograd): one training step's worth
  paged    keys and values in pages of a cache; `new` tokens of each sequence (binding)
  append   rotation of q and k, and k and v into their pages (binding)

Queries and keys are multiples of 1/16 below 16.  K-TanH jumps at the ends of its intervals (by up to 0.016),
and such values make every q . k exact in Float32 whatever the order of its sum, so that all sides see the
same interval.  Each head has its own spread: scores of a standard deviation between 1 and 6 before the cap,
as between a head that looks everywhere and one that looks at few tokens.
"""
import math
import random

import torch

own = False

# ------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # The smallest call: one short prompt through a small layer.
        {"name": "attend_short", "kind": "attend", "docs": 1, "tokens": 100, "heads": 8, "kv_heads": 8, "dim": 64,
         "cap": 30.0, "causal": True, "window": 0, "intervals": 32, "ragged": 0},
        # Sixteen prompts of different lengths in one call, shared heads.
        {"name": "attend_docs", "kind": "attend", "docs": 16, "tokens": 8192, "heads": 32, "kv_heads": 8, "dim": 128,
         "cap": 50.0, "causal": True, "window": 0, "intervals": 32, "ragged": 1},
        # A layer with a sliding window over one long document.
        {"name": "attend_window", "kind": "attend", "docs": 1, "tokens": 16384, "heads": 16, "kv_heads": 8, "dim": 64,
         "cap": 50.0, "causal": True, "window": 1024, "intervals": 64, "ragged": 0},
        # One long prompt.
        {"name": "attend_long", "kind": "attend", "docs": 1, "tokens": 16384, "heads": 32, "kv_heads": 8, "dim": 128,
         "cap": 50.0, "causal": True, "window": 0, "intervals": 32, "ragged": 0},
        # A training step of a small model on a few odd documents, bidirectional.
        {"name": "train_small", "kind": "train", "docs": 4, "tokens": 1021, "heads": 8, "kv_heads": 2, "dim": 64,
         "cap": 30.0, "causal": False, "window": 0, "intervals": 32, "ragged": 2},
        # A training step on a sequence of packed documents.
        {"name": "train_docs", "kind": "train", "docs": 6, "tokens": 8192, "heads": 32, "kv_heads": 8, "dim": 128,
         "cap": 50.0, "causal": True, "window": 0, "intervals": 32, "ragged": 3},
        # One token for one user.
        {"name": "decode_one", "kind": "paged", "docs": 1, "longest": 777, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "cap": 50.0, "window": 0, "intervals": 32, "ragged": 0},
        # One token for each of 64 users, whose texts have all lengths.
        {"name": "decode_batch", "kind": "paged", "docs": 64, "longest": 8192, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "cap": 50.0, "window": 0, "intervals": 32, "ragged": 4},
        # One token each behind two very long texts.
        {"name": "decode_long", "kind": "paged", "docs": 2, "longest": 131071, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "cap": 50.0, "window": 0, "intervals": 64, "ragged": 0},
        # A piece of a prompt for each of four users, behind what is cached of it.
        {"name": "prompt_piece", "kind": "paged", "docs": 4, "longest": 6000, "new": 512, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "cap": 50.0, "window": 0, "intervals": 32, "ragged": 5},
        # The new token of each of 64 users into the cache ...
        {"name": "append_step", "kind": "append", "docs": 64, "tokens": 64, "longest": 8192, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "interleaved": False, "ragged": 6},
        # ... and the prompts of sixteen.
        {"name": "append_prompts", "kind": "append", "docs": 16, "tokens": 16384, "longest": 4096, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "interleaved": False, "ragged": 7},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


_HEADS = ((8, 8), (8, 2), (16, 8), (12, 4), (32, 8), (40, 8), (5, 1))


def draw(rng):
    kind = rng.choice(("attend", "attend", "train", "train", "paged", "paged", "paged", "append"))
    heads, kv_heads = rng.choice(_HEADS)
    case = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "dim": rng.choice((64, 128, 128)),
            "ragged": rng.randrange(1, 1 << 30)}
    if kind == "append":
        case |= {"docs": _log_int(rng, 1, 64), "page": rng.choice((8, 16, 64, 256)), "interleaved": rng.random() < 0.3}
        case["tokens"] = case["docs"] if rng.random() < 0.5 else _log_int(rng, case["docs"], 16384)
        case["longest"] = case["tokens"] + _log_int(rng, 1, 8192)
        while case["docs"] * case["longest"] * kv_heads * case["dim"] > 1 << 28:
            case["longest"] = case["tokens"] + (case["longest"] - case["tokens"]) // 2
            case["docs"] = max(1, case["docs"] // 2)
            case["tokens"] = max(case["docs"], case["tokens"] // 2)
        return case
    case |= {"cap": rng.choice((20.0, 50.0)), "intervals": rng.choice((32, 32, 64)),
             "window": rng.choice((0, 0, 0, _log_int(rng, 16, 4096)))}
    if kind == "paged":
        case |= {"docs": _log_int(rng, 1, 96), "longest": _log_int(rng, 16, 131072), "page": rng.choice((8, 16, 64, 256)),
                 "new": 1 if rng.random() < 0.7 else _log_int(rng, 2, 512)}
        case["new"] = min(case["new"], case["longest"])
        while case["docs"] * case["longest"] * kv_heads * case["dim"] > 1 << 29 or case["docs"] * case["new"] * case["longest"] > 1 << 24:
            case["longest"] = max(case["new"], case["longest"] // 2)
            case["docs"] = max(1, case["docs"] // 2)
        return case
    case |= {"docs": _log_int(rng, 1, 32), "causal": rng.random() < 0.75}
    case["tokens"] = max(case["docs"], _log_int(rng, 16, 16384 if kind == "attend" else 8192))
    while sum(n * n for n in _lengths(case)) * heads > (1 << 31 if kind == "attend" else 1 << 29):
        case["tokens"] = max(case["docs"], case["tokens"] * 3 // 4)
    return case


def _lengths(case):
    """attend, train, append: how many of the tokens each document has.  paged: how many each sequence has in all."""
    rng, docs = random.Random(case["ragged"]), case["docs"]
    if case["kind"] == "paged":
        low = max(case["new"], 1)
        if not case["ragged"]:
            return [case["longest"]] * docs
        return [low + int((case["longest"] - low) * rng.random()) for _ in range(docs)]
    tokens = case["tokens"]
    if not case["ragged"] or tokens == docs:
        return [tokens // docs + (i < tokens % docs) for i in range(docs)]
    cuts = sorted(rng.sample(range(1, tokens), docs - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [tokens])]


def _cached(case):
    """append: how many tokens each sequence has in the cache before the call."""
    rng = random.Random(case["ragged"] + 1)
    return [int((case["longest"] - n) * rng.random()) if case["longest"] > n else 0 for n in _lengths(case)]


def _seen(rows, keys, causal, window):
    """Pairs of a query and a key that it sees, `rows` queries at the end of `keys` keys."""
    seen = 0
    for i in range(rows) if window or (causal and rows > keys) else ():
        at = i + keys - rows
        seen += max(0, (min(at + 1, keys) if causal else keys) - (max(0, at + 1 - window) if window else 0))
    if window or (causal and rows > keys):
        return seen
    return rows * keys - (rows * (rows - 1) // 2 if causal else 0)


# ------------------------------------------------------------------------------------------ inputs


def _offsets(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _grid(gen, shape, heads):
    """Normal values, head by head with a spread of their own, as multiples of 1/16 below 16."""
    spread = torch.rand((heads, 1), generator=gen, device="cuda").mul_(math.log(6.0) / 2).exp_()
    x = torch.randn(shape, generator=gen, device="cuda") * spread
    return (x * 16).round_().clamp_(-255, 255).div_(16).bfloat16()


def _normal(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda").bfloat16()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    heads, kv_heads, dim, kind = case["heads"], case["kv_heads"], case["dim"], case["kind"]
    lengths = _lengths(case)
    state = {"case": case, "scale": dim ** -0.5}
    if kind in ("attend", "train"):
        tokens = case["tokens"]
        state["q"] = _grid(gen, (tokens, heads, dim), heads)
        state["k"] = _grid(gen, (tokens, kv_heads, dim), kv_heads)
        state["v"] = _normal(gen, (tokens, kv_heads, dim))
        state["offsets"], state["docs"] = _int32(_offsets(lengths)), lengths
        if kind == "train":
            state["do"] = _normal(gen, (tokens, heads, dim))
            for name in "qkv":
                state[name].requires_grad_()
        return state
    page, docs = case["page"], case["docs"]
    most = -(-case["longest"] // page)
    count = docs * most + 3                      # a few pages of the cache belong to nobody
    state["pages"] = torch.randperm(count, generator=gen, device="cuda")[:docs * most].view(docs, most).int()
    if kind == "paged":
        state["k_cache"] = _grid(gen, (count, page, kv_heads, dim), kv_heads)
        state["v_cache"] = _normal(gen, (count, page, kv_heads, dim))
        state["q"] = _grid(gen, (docs * case["new"], heads, dim), heads)
        state["lengths"], state["docs"] = _int32(lengths), lengths
        state["offsets"] = None if case["new"] == 1 else _int32([i * case["new"] for i in range(docs + 1)])
        return state
    tokens = case["tokens"]
    state["k_cache"], state["v_cache"] = (_normal(gen, (count, page, kv_heads, dim)) for _ in range(2))
    state["q"], state["k"], state["v"] = (_normal(gen, (tokens, h, dim)) for h in (heads, kv_heads, kv_heads))
    before = _cached(case)
    state["before"] = _int32(before)
    state["offsets"] = None if lengths == [1] * docs else _int32(_offsets(lengths))
    state["sequence"] = torch.repeat_interleave(torch.arange(docs), torch.tensor(lengths)).cuda()
    state["position"] = torch.cat([torch.arange(a, a + n) for a, n in zip(before, lengths)]).cuda()
    angle = torch.outer(torch.arange(case["longest"], dtype=torch.float64),
                        10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim))
    state["cos"], state["sin"] = angle.cos().float().cuda(), angle.sin().float().cuda()
    return state


# -------------------------------------------------------------------------------------------- pass


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"attend": _plain_attend, "train": _plain_train, "paged": _plain_paged, "append": _plain_append}[kind](state)
    from paper_1909_07729_amd import autograd, binding
    if kind == "append":
        q = binding.kcap_append(state["q"], state["k"], state["v"], state["k_cache"], state["v_cache"], state["pages"],
                                state["before"], state["offsets"], cos=state["cos"], sin=state["sin"],
                                interleaved=case["interleaved"])
        return {"q": q, "k_cache": state["k_cache"], "v_cache": state["v_cache"]}
    asked = {"cap": case["cap"], "scale": state["scale"], "window": case["window"]}
    if kind == "paged":
        paged = binding.kcap_attention_paged if case["intervals"] == 32 else binding.kcap_attention64_paged
        return {"o": paged(state["q"], state["k_cache"], state["v_cache"], state["pages"], state["lengths"],
                           state["offsets"], **asked)}
    asked["causal"] = case["causal"]
    if kind == "attend":
        attend = binding.kcap_attention if case["intervals"] == 32 else binding.kcap_attention64
        o, lse = attend(state["q"], state["k"], state["v"], state["offsets"], **asked)
        return {"o": o, "lse": lse}
    o = autograd.kcap_attention(state["q"], state["k"], state["v"], state["offsets"], intervals=case["intervals"], **asked)
    dq, dk, dv = torch.autograd.grad(o, (state["q"], state["k"], state["v"]), state["do"])
    return {"o": o.detach(), "dq": dq, "dk": dk, "dv": dv}


# ------------------------------------------------------------------------------------ the plain form

# K-TanH's table, (E_t, r_t, b_t) by index t: Table 1 of the paper, and what its fit gives for 64 intervals.
_E32 = [126] * 8 + [125] * 9 + [126] * 15
_R32 = [2, 4, 4, 4, 6, 6, 6, 6, 1, 0, 0, 0, 0, 0, 0, 0, 0, 1, 1, 1, 1, 1, 1, 1, 0, 1, 1, 1, 2, 2, 2, 4]
_B32 = [119, 122, 123, 123, 126, 126, 126, 126, 1, -4, -6, -7, -10, -12, -15, -18,
        112, -4, -1, 2, 3, 4, 4, 4, 65, 72, 73, 73, 88, 89, 89, 110]
_E64 = [126] * 16 + [125] * 18 + [126] * 30
_R64 = [2, 3, 2, 5, 5, 4, 4, 7, 6, 6, 6, 6, 6, 6, 6, 5, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0,
        0, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 0, 1, 1, 1, 1, 1, 1, 2, 2, 2, 2, 2, 2, 3, 2, 3]
_B64 = [119, 120, 118, 123, 124, 123, 123, 126, 126, 126, 126, 126, 126, 126, 126, 124,
        0, -3, -4, -5, -5, -6, -7, -8, -9, -10, -11, -13, -14, -15, -17, -18,
        111, 119, -5, -3, -1, 0, 1, 2, 3, 4, 4, 4, 4, 4, 4, 3,
        66, 70, 72, 73, 73, 73, 73, 87, 88, 89, 89, 89, 89, 102, 88, 103]


def _lines(intervals):
    """(slope, intercept) of K on the intervals from 0.125 to 16, by the low bits of exponent and mantissa."""
    wide = intervals == 64
    table = list(zip(*((_E64, _R64, _B64) if wide else (_E32, _R32, _B32))))
    each = 16 if wide else 8
    lines = [(0.0, 1.0)] * (8 * each)
    for exponent in range(124, 132):
        for m in range(each):
            E, r, b = table[(exponent & 3) * each + m]
            at = (exponent & 7) * each + m
            if exponent == 124:
                lines[at] = (1.0, 0.0)
            elif exponent <= 128:
                lines[at] = (2.0 ** (E - exponent - r), 2.0 ** (E - 127) * (1.0 - 2.0 ** -r + b / 128))
    return lines


_ON_GPU = {}


def _k_f32(x, intervals):
    if intervals not in _ON_GPU:        # K's constants, as a program has them on the GPU
        _ON_GPU[intervals] = torch.tensor(_lines(intervals), device="cuda").unbind(1)
    slope, intercept = _ON_GPU[intervals]
    mag = x.abs()
    at = mag.clamp(0.125, 8.0).view(torch.int32) >> (19 if intervals == 64 else 20)
    at &= 127 if intervals == 64 else 63
    return torch.copysign(slope[at] * mag.clamp(max=8.0) + intercept[at], x)


def _masked(y, rows, keys, causal, window):
    """Scores of `rows` queries at the end of `keys` keys, -infinity where a query does not see a key."""
    if not causal and not window:
        return y
    at = torch.arange(rows, device=y.device)[:, None] + (keys - rows)
    key = torch.arange(keys, device=y.device)[None, :]
    hidden = key > at if causal else torch.zeros_like(key > at)
    if window:
        hidden = hidden | (key <= at - window)
    return y.masked_fill(hidden, -math.inf)


def _weights(q, k, case, scale, causal):
    """K of the scores, the softmax weights and the log-sums; q [heads, rows, dim], k [heads, keys, dim]."""
    t = _k_f32(torch.matmul(q, k.transpose(1, 2)) * (scale / case["cap"]), case["intervals"])
    y = _masked(t * case["cap"], q.shape[1], k.shape[1], causal, case["window"])
    top = y.amax(-1, keepdim=True).clamp(min=-3e38)
    p = (y - top).exp()
    total = p.sum(-1, keepdim=True)
    return t, p / total.clamp(min=1e-38), (top + total.log()).squeeze(-1)


def _heads_at_once(rows, keys, heads):
    """A divisor of the heads such that a piece of the scores stays in the hundreds of MB."""
    most = max(1, (1 << 27) // max(1, rows * keys))
    return max(h for h in range(1, heads + 1) if heads % h == 0 and h <= most)


def _plain_rows(q, k, v, case, scale, causal):
    """Outputs [rows, heads, dim] and log-sums [heads, rows] of one document, all in Float32."""
    group = q.shape[1] // k.shape[1]
    q, k, v = q.transpose(0, 1), *(t.transpose(0, 1).repeat_interleave(group, 0) for t in (k, v))
    h = _heads_at_once(q.shape[1], k.shape[1], q.shape[0])

    def piece(q, k, v):
        _, p, lse = _weights(q, k, case, scale, causal)
        return torch.matmul(p, v), lse
    parts = [piece(*t) for t in zip(q.split(h), k.split(h), v.split(h))]
    return torch.cat([p[0] for p in parts]).transpose(0, 1), torch.cat([p[1] for p in parts])


def _plain_attend(state):
    case = state["case"]
    parts = [_plain_rows(q.float(), k.float(), v.float(), case, state["scale"], case["causal"])
             for q, k, v in zip(*(state[n].split(state["docs"]) for n in "qkv"))]
    return {"o": torch.cat([p[0] for p in parts]).bfloat16(), "lse": torch.cat([p[1] for p in parts], 1)}


def _plain_grads(q, k, v, do, case, scale):
    group, kv_heads = q.shape[1] // k.shape[1], k.shape[1]
    q, do = (t.transpose(0, 1).float() for t in (q, do))
    k, v = (t.transpose(0, 1).float().repeat_interleave(group, 0) for t in (k, v))
    h = _heads_at_once(q.shape[1], k.shape[1], q.shape[0])

    def piece(q, k, v, do):
        t, p, _ = _weights(q, k, case, scale, case["causal"])
        o = torch.matmul(p, v)
        dv = torch.matmul(p.transpose(1, 2), do)
        ds = (torch.matmul(do, v.transpose(1, 2)) - (o * do).sum(-1, keepdim=True)) * p * (1.0 - t * t) * scale
        return o, torch.matmul(ds, k), torch.matmul(ds.transpose(1, 2), q), dv
    parts = [piece(*t) for t in zip(q.split(h), k.split(h), v.split(h), do.split(h))]
    o, dq, dk, dv = (torch.cat([p[i] for p in parts]) for i in range(4))
    dk, dv = (t.unflatten(0, (kv_heads, group)).sum(1) for t in (dk, dv))
    return [t.transpose(0, 1).bfloat16() for t in (o, dq, dk, dv)]


def _plain_train(state):
    with torch.no_grad():
        parts = [_plain_grads(*t, state["case"], state["scale"])
                 for t in zip(*(state[n].split(state["docs"]) for n in ("q", "k", "v", "do")))]
        return dict(zip(("o", "dq", "dk", "dv"), (torch.cat([p[i] for p in parts]) for i in range(4))))


def _from_pages(cache, pages, length):
    return cache[pages[:-(-length // cache.shape[1])].long()].flatten(0, 1)[:length]


def _plain_paged(state):
    case = state["case"]
    parts = [_plain_rows(q.float(), *(_from_pages(state[n], pages, n_keys).float() for n in ("k_cache", "v_cache")),
                         case, state["scale"], True)[0]
             for q, pages, n_keys in zip(state["q"].split(case["new"]), state["pages"], state["docs"])]
    return {"o": torch.cat(parts).bfloat16()}


def _rotated(x, cos, sin, interleaved):
    """Pairs (x_i, x_{i+dim/2}), or (x_{2i}, x_{2i+1}) where interleaved, turned by their angles."""
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)
    cos, sin = cos[:, None, :], sin[:, None, :]
    turned = a * cos - b * sin, b * cos + a * sin
    return torch.stack(turned, -1).flatten(-2) if interleaved else torch.cat(turned, -1)


def _plain_append(state):
    case, at = state["case"], state["position"]
    cos, sin = state["cos"][at], state["sin"][at]
    page, slot = state["pages"][state["sequence"], at // case["page"]].long(), at % case["page"]
    q, k = (_rotated(state[n].float(), cos, sin, case["interleaved"]).bfloat16() for n in "qk")
    state["k_cache"][page, slot] = k
    state["v_cache"][page, slot] = state["v"]
    return {"q": q, "k_cache": state["k_cache"], "v_cache": state["v_cache"]}


# -------------------------------------------------------------------------------------------- work


def work(case):
    heads, kv_heads, dim, kind = case["heads"], case["kv_heads"], case["dim"], case["kind"]
    lengths = _lengths(case)
    if kind == "append":  # q in and out, k and v in and into the cache; the angles of each token
        return {"bytes": case["tokens"] * (4 * heads + 8 * kv_heads + 4) * dim, "flops": case["tokens"] * 3 * (heads + kv_heads) * dim}
    if kind == "paged":
        new, window = case["new"], case["window"]
        pairs = sum(_seen(new, n, True, window) for n in lengths)
        keys = sum(min(n, window + new - 1) if window else n for n in lengths)
        return {"bytes": 4 * dim * (kv_heads * keys + heads * case["docs"] * new), "flops": 4 * dim * heads * pairs}
    pairs = sum(_seen(n, n, case["causal"], case["window"]) for n in lengths)
    tokens = case["tokens"]
    if kind == "attend":  # q, k, v in; o and the log-sums out
        return {"bytes": tokens * (4 * dim * (heads + kv_heads) + 4 * heads), "flops": 4 * dim * heads * pairs}
    # two products forward, five backward; q, k, v, do in, o, dq, dk, dv out
    return {"bytes": 8 * dim * tokens * (heads + kv_heads), "flops": 14 * dim * heads * pairs}


# ------------------------------------------------------------------------------------------- exact


def _k64(x, intervals):
    """Algorithm 1 of the paper on doubles: thresholds, index, shift and add, with nothing cut off."""
    bits = 4 if intervals == 64 else 3
    mag = x.abs()
    _, exponent = torch.frexp(mag.clamp(0.25, 3.99))
    exponent = exponent - 1
    fraction = mag / torch.pow(2.0, exponent.double()) - 1.0
    t = (((exponent + 127) & 3) << bits) | (fraction * 2 ** bits).floor().long().clamp(0, 2 ** bits - 1)
    E, r, b = (torch.tensor(u, dtype=torch.float64, device=x.device)[t] for u in ((_E64, _R64, _B64) if intervals == 64 else (_E32, _R32, _B32)))
    out = torch.pow(2.0, E - 127.0) * (1.0 + fraction * torch.pow(2.0, -r) + b / 128.0)
    out = torch.where(mag < 0.25, mag, torch.where(mag >= 4.0, torch.ones_like(mag), out))
    return torch.sign(x) * out


def _exact_head(q, k, v, do, case, scale, causal):
    """One head of one document, in doubles: (o, lse), and with `do` the gradients behind them."""
    rows, keys = q.shape[0], k.shape[0]
    t = _k64(q @ k.T * scale / case["cap"], case["intervals"])
    place = torch.arange(keys - rows, keys, device=q.device).view(-1, 1) - torch.arange(keys, device=q.device)
    seen = torch.ones_like(place, dtype=torch.bool)
    if causal:
        seen &= place >= 0
    if case["window"]:
        seen &= place < case["window"]
    e = torch.exp(case["cap"] * t) * seen                   # scores are bounded: no maximum needed
    total = e.sum(1)
    p = e / torch.where(total > 0, total, torch.ones_like(total))[:, None]
    o = p @ v
    if do is None:
        return o, torch.log(total)
    dp = do @ v.T
    ds = p * (dp - (p * dp).sum(1, keepdim=True)) * (1.0 - t ** 2)
    return o, scale * (ds @ k), scale * (ds.T @ q), p.T @ do


def exact(case, seed):
    kind, heads, kv_heads = case["kind"], case["heads"], case["kv_heads"]
    lengths = _lengths(case)
    if kind != "append":
        pairs = sum(case.get("new", n) * n for n in lengths) * heads
        if pairs > 2e10:            # beyond about 20 seconds
            return None
    state = prepare(case, seed)
    with torch.no_grad():
        if kind == "append":
            at = state["position"]
            cos, sin = (state[n].double()[at][:, None, :] for n in ("cos", "sin"))
            made = {}
            for name in "qk":
                x = state[name].double()
                half = x.shape[-1] // 2
                pairs = x.unflatten(-1, (half, 2)) if case["interleaved"] else x.unflatten(-1, (2, half)).transpose(-1, -2)
                z = torch.view_as_complex(pairs.contiguous()) * torch.complex(cos, sin)
                z = torch.view_as_real(z)
                made[name] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            caches = [state[n].double() for n in ("k_cache", "v_cache")]
            for cache, rows in zip(caches, (made["k"], state["v"].double())):
                flat = cache.flatten(0, 1)
                flat[state["pages"][state["sequence"], at // case["page"]].long() * case["page"] + at % case["page"]] = rows
            return {"q": made["q"], "k_cache": caches[0], "v_cache": caches[1]}
        group = heads // kv_heads
        outs = []
        start = 0
        for doc, n in enumerate(lengths):
            if kind == "paged":
                page = case["page"]
                rows = [int(p) for p in state["pages"][doc, :-(-n // page)]]
                k, v = (torch.cat([state[c][p] for p in rows])[:n].double() for c in ("k_cache", "v_cache"))
                q, do = state["q"][doc * case["new"]:(doc + 1) * case["new"]].double(), None
            else:
                q, k, v = (state[c][start:start + n].double() for c in "qkv")
                do = state["do"][start:start + n].double() if kind == "train" else None
                start += n
            outs.append([_exact_head(q[:, h], k[:, h // group], v[:, h // group], None if do is None else do[:, h],
                                     case, state["scale"], True if kind == "paged" else case["causal"])
                         for h in range(heads)])
        o = torch.cat([torch.stack([h[0] for h in doc], 1) for doc in outs])
        if kind == "paged":
            return {"o": o}
        if kind == "attend":
            return {"o": o, "lse": torch.cat([torch.stack([h[1] for h in doc]) for doc in outs], 1)}
        dq = torch.cat([torch.stack([h[1] for h in doc], 1) for doc in outs])
        dk, dv = (torch.cat([torch.stack([h[i] for h in doc], 1).unflatten(1, (kv_heads, group)).sum(2) for doc in outs])
                  for i in (2, 3))
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
