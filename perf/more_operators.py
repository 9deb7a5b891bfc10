"""Products and checkpoints in 8 bits and the choice of the next token, as cases that can be timed and checked.

A case is a plain dict.  ``listed()`` names a few, ``draw(rng)`` makes more of the same ranges,
``prepare(case, seed)`` builds what a program has in hand before the call, ``run(state)`` is one pass,
``work(case)`` the bytes and operations that the pass cannot do without, ``exact(case, seed)`` the same
outputs in 64 bits.  With ``own`` false ``run`` computes them with elementary torch operations, with ``own``
true through the library.

Kinds of case
  linear   tokens to 8-bit integers, each with a scale of its own, behind an activation or none, and their
           product with weights in 8 bits that have a scale for each output channel (binding)
  product  the same product of tokens that are in 8 bits already (binding)
  keep     one training step through an activation that keeps its input in 8 bits for the backward pass:
           the output, and the gradient (autograd)
  back     that backward pass alone, which also rebuilds the activation's output for the gradient of the
           weights behind it (binding)
  sample   one token of each row of logits by temperature, top-k, top-p and min-p from given uniform
           numbers, the logits capped through K-TanH or not (binding)

Integers of a row of values x: s = max|x| / 127, code = round(x * (127 / max|x|)), both in Float32 operations, to
nearest even.  A checkpoint has a scale for each 128 consecutive values, and stands for code * s, rounded to the
tensor's type.  The activations are the library's: their operations are Float32, one rounding each.

Sampling ranks the tokens by logit, the lowest index first where they are equal, with weights exp((logit - max) / T).
top-k keeps the first k; top-p those of them whose predecessors weigh less than p of these; min-p those whose weight
is at least min_p of the largest.  The token is the first whose weight and its predecessors' exceed u of all kept.
"""
import math
import random

import torch

own = False

GROUP = 128             # values of a checkpoint that share a scale

# ------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # One token for one user through a square layer: the time of a call, and of the weights' way to the chip.
        {"name": "linear_token", "kind": "linear", "tokens": 1, "inner": 4096, "outer": 4096, "type": "bf16", "out": "bf16",
         "bias": False, "activation": "", "intervals": 32, "apart": 0},
        # One token for each of 64 users through the wide half of an MLP.
        {"name": "linear_users", "kind": "linear", "tokens": 64, "inner": 4096, "outer": 16384, "type": "bf16", "out": "bf16",
         "bias": True, "activation": "", "intervals": 32, "apart": 0},
        # A short prompt through a layer of odd sizes, from Float32 rows that are columns of a wider tensor.
        {"name": "linear_odd", "kind": "linear", "tokens": 777, "inner": 1001, "outer": 2003, "type": "f32", "out": "f32",
         "bias": True, "activation": "swish", "intervals": 64, "apart": 23},
        # Prompts of 8192 tokens in all through the narrow half of an MLP, its GELU in front.
        {"name": "linear_prompts", "kind": "linear", "tokens": 8192, "inner": 16384, "outer": 4096, "type": "bf16", "out": "bf16",
         "bias": False, "activation": "gelu", "intervals": 32, "apart": 0},
        # One of several products of the same tokens.
        {"name": "product_prompts", "kind": "product", "tokens": 2048, "inner": 4096, "outer": 6144, "type": "bf16", "out": "bf16",
         "bias": False, "activation": "", "intervals": 32, "apart": 0},
        # The logits of a few tokens, kept in Float32.
        {"name": "product_logits", "kind": "product", "tokens": 24, "inner": 2048, "outer": 50000, "type": "bf16", "out": "f32",
         "bias": False, "activation": "", "intervals": 32, "apart": 0},
        # A training step of a small model: about a thousand tokens of packed documents.
        {"name": "keep_small", "kind": "keep", "count": 1021 * 1024, "type": "bf16", "activation": "gelu", "intervals": 32},
        # A training step's MLP of 8192 tokens.
        {"name": "keep_mlp", "kind": "keep", "count": 8192 * 16384, "type": "bf16", "activation": "gelu", "intervals": 32},
        # The backward pass of a layer in Float32, an odd number of values.
        {"name": "back_odd", "kind": "back", "count": 4001 * 4999, "type": "f32", "activation": "swish", "intervals": 64},
        # ... and of a wide one.
        {"name": "back_mlp", "kind": "back", "count": 4096 * 16384, "type": "bf16", "activation": "gelu", "intervals": 32},
        # The next token of one user.
        {"name": "sample_one", "kind": "sample", "rows": 1, "vocabulary": 32000, "type": "f32", "spread": 3.0, "each": False,
         "temperature": 0.8, "top_k": 50, "top_p": 0.95, "min_p": 0.0, "cap": 0.0, "intervals": 32, "masked": 0.0},
        # The next token of 64 users, each with settings of their own, from capped logits.
        {"name": "sample_users", "kind": "sample", "rows": 64, "vocabulary": 131072, "type": "bf16", "spread": 4.0, "each": True,
         "temperature": 1.0, "top_k": 0, "top_p": 0.9, "min_p": 0.02, "cap": 30.0, "intervals": 32, "masked": 0.1},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _side(rng):
    """An inner or outer size: mostly a multiple of 64, sometimes any."""
    n = _log_int(rng, 64, 16384)
    return n if rng.random() < 0.3 else max(64, n // 64 * 64)


def draw(rng):
    kind = rng.choice(("linear", "linear", "linear", "product", "keep", "back", "sample", "sample"))
    case = {"kind": kind, "intervals": rng.choice((32, 32, 64))}
    if kind in ("linear", "product"):
        case |= {"tokens": _log_int(rng, 1, 8192), "inner": _side(rng), "outer": _side(rng), "type": rng.choice(("bf16", "bf16", "f32")),
                 "out": rng.choice(("bf16", "bf16", "f32")), "bias": rng.random() < 0.3,
                 "activation": rng.choice(("", "gelu", "swish")) if kind == "linear" else "",
                 "apart": _log_int(rng, 1, 100) if kind == "linear" and rng.random() < 0.3 else 0}
        while case["tokens"] * case["inner"] * case["outer"] > 1 << 38:
            case["tokens"] //= 2
        return case
    if kind in ("keep", "back"):
        return case | {"count": _log_int(rng, 1000, 1 << 26), "type": rng.choice(("bf16", "bf16", "f32")),
                       "activation": rng.choice(("gelu", "swish"))}
    case |= {"rows": _log_int(rng, 1, 256), "vocabulary": _log_int(rng, 64, 262144), "type": rng.choice(("bf16", "f32")),
             "spread": rng.uniform(0.5, 6.0), "each": rng.random() < 0.6, "temperature": rng.choice((0.0, 0.5, 0.8, 1.0, 1.3)),
             "top_k": rng.choice((0, 0, 1, 20, 50, 1000)), "top_p": rng.choice((1.0, 0.95, 0.9, 0.5)),
             "min_p": rng.choice((0.0, 0.0, 0.02, 0.1)), "cap": rng.choice((0.0, 0.0, 30.0)), "masked": rng.choice((0.0, 0.0, 0.1, 0.9))}
    while case["rows"] * case["vocabulary"] > 1 << 23:
        case["rows"] = max(1, case["rows"] // 2)
    return case


# ------------------------------------------------------------------------------------------ inputs

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _uniform(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda")


def _by(x, y):
    """The quotient by a number, correctly rounded (torch's own division by a Python number takes the reciprocal)."""
    return x / torch.full_like(x, y)


def _rows_in_8_bits(x):
    """(codes, scales) of Float32 rows; rows of codes begin at multiples of 16 bytes, as the library's own do."""
    top = x.abs().amax(1, keepdim=True)
    room = torch.zeros((x.shape[0], -(-x.shape[1] // 16) * 16), dtype=torch.int8, device=x.device)
    codes = room[:, :x.shape[1]]
    codes.copy_(_codes(x, top))
    return codes, _by(top, 127.0).squeeze(1)


def _codes(x, top):
    """Integers of Float32 values under the largest magnitude that they share."""
    return (x * (torch.full_like(top, 127.0) / top.clamp(min=1e-30))).round()


def _tokens(gen, rows, inner):
    """Rows as they leave a norm: one channel in 64 is some ten times the others, and tokens differ in size."""
    loud = torch.where(_uniform(gen, 1, inner) < 1 / 64, 10.0, 1.0)
    return _normal(gen, rows, inner) * loud * (1.0 + _uniform(gen, rows, 1))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state, kind = {"case": case}, case["kind"]
    if kind in ("linear", "product"):
        tokens, inner, outer = case["tokens"], case["inner"], case["outer"]
        x = _tokens(gen, tokens, inner + case["apart"]).to(_TYPES[case["type"]])[:, :inner]
        weight = _normal(gen, outer, inner) * ((0.5 + _uniform(gen, outer, 1)) / math.sqrt(inner))
        state["weight"], state["weight_scale"] = _rows_in_8_bits(weight)
        state["bias"] = _normal(gen, outer) if case["bias"] else None
        if kind == "linear":
            state["x"] = x
        else:
            state["tokens"], state["token_scale"] = _rows_in_8_bits(x.float())
        return state
    if kind in ("keep", "back"):
        # what comes from the product in front: normal, of different size from place to place
        count = case["count"]
        size = (2.0 * _uniform(gen, -(-count // 1024))).repeat_interleave(1024)[:count] + 0.5
        x = (_normal(gen, count) * size).to(_TYPES[case["type"]])
        state["dy"] = _normal(gen, count).to(x.dtype)
        if kind == "keep":
            state["x"] = x.requires_grad_()
        else:
            state["codes"], state["scales"] = _checkpoint(x.float())
        return state
    rows, vocabulary = case["rows"], case["vocabulary"]
    logits = _normal(gen, rows, vocabulary) * case["spread"]
    if case["masked"]:      # tokens that a grammar forbids; never all of them
        forbidden = _uniform(gen, rows, vocabulary) < case["masked"]
        forbidden[:, 0] = False
        logits.masked_fill_(forbidden, -math.inf)
    state["logits"] = logits.to(_TYPES[case["type"]])
    state["uniform"] = _uniform(gen, rows)
    for name in ("temperature", "top_k", "top_p", "min_p"):
        state[name] = case[name]
    if case["each"]:        # settings that differ from user to user, some of them without a filter, some greedy
        def some(values, dtype=torch.float32):
            return torch.tensor(values, dtype=dtype, device="cuda")[torch.randint(len(values), (rows,), generator=gen, device="cuda")]
        state["temperature"] = some([case["temperature"]] * 6 + [0.0, 1.0])
        state["top_k"] = some([case["top_k"]] * 6 + [0, 40], torch.int32)
        state["top_p"] = some([case["top_p"]] * 6 + [1.0, 0.8])
        state["min_p"] = some([case["min_p"]] * 6 + [0.0, 0.05])
    return state


# -------------------------------------------------------------------------------------------- pass


def run(state):
    case = state["case"]
    kind, wide = case["kind"], case["intervals"] == 64
    if not own:
        return {"linear": _plain_linear, "product": _plain_product, "keep": _plain_keep, "back": _plain_back,
                "sample": _plain_sample}[kind](state)
    from paper_1909_07729_amd import autograd, binding
    if kind == "linear":
        linear = binding.kq8_linear64 if wide else binding.kq8_linear
        return {"out": linear(state["x"], state["weight"], state["weight_scale"], state["bias"],
                              activation=case["activation"] or None, out_dtype=_TYPES[case["out"]])}
    if kind == "product":
        return {"out": binding.kq8_product(state["tokens"], state["token_scale"], state["weight"], state["weight_scale"],
                                           state["bias"], out_dtype=_TYPES[case["out"]])}
    if kind == "keep":
        activation = autograd.kgelu if case["activation"] == "gelu" else autograd.kswish
        y = activation(state["x"], intervals=case["intervals"], keep=8)
        dx, = torch.autograd.grad(y, state["x"], state["dy"])
        return {"y": y.detach(), "dx": dx}
    if kind == "back":
        name = f"k{case['activation']}{'64' if wide else ''}{'_f32' if case['type'] == 'f32' else ''}_keep8_backward"
        dx, y = getattr(binding, name)(state["dy"], state["codes"], state["scales"], rebuild=True)
        return {"dx": dx, "y": y}
    sample = binding.ksample64 if wide else binding.ksample
    return {"tokens": sample(state["logits"], state["uniform"], temperature=state["temperature"], top_k=state["top_k"],
                             top_p=state["top_p"], min_p=state["min_p"], cap=case["cap"])}


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

_ON_GPU = {}


def _table(intervals):
    """Base and shift of each interval, as Float32 patterns: the output's are base + (mantissa >> shift)."""
    if intervals not in _ON_GPU:        # K's constants, as a program has them on the GPU
        E, r, b = (_E64, _R64, _B64) if intervals == 64 else (_E32, _R32, _B32)
        _ON_GPU[intervals] = (torch.tensor([(e << 23) + (o << 16) for e, o in zip(E, b)], dtype=torch.int32, device="cuda"),
                              torch.tensor(r, dtype=torch.int32, device="cuda"))
    return _ON_GPU[intervals]


def _k(x, intervals):
    """K-TanH of Float32 values, in their type: Algorithm 1 on the bit fields."""
    base, shift = _table(intervals)
    bits = x.view(torch.int32)
    mag = bits & 0x7FFFFFFF
    t = (mag >> (19 if intervals == 64 else 20)) & (intervals - 1)
    out = base[t] + ((mag & 0x7FFFFF) >> shift[t])
    out = torch.where(mag >= 0x40800000, 0x3F800000, torch.where(mag < 0x3E800000, mag, out))
    return (out | (bits & -0x80000000)).view(torch.float32)


def _k_as(x, dtype, intervals):
    """K of a Float32 argument for tensors of `dtype`: BFloat16 ones round the argument, and K's result is one."""
    if dtype == torch.float32:
        return _k(x, intervals)
    return (_k(x.to(dtype).float(), intervals).view(torch.int32) & -0x10000).view(torch.float32)


_A, _A3, _C = 0.044715, 0.134145, 0.7978845608028654


def _inner(x, activation, dtype, intervals):
    """What the activation and its slope are made of: K of GELU's argument, or Swish's Sigmoid."""
    if activation == "gelu":
        return _k_as((x + x * x * x * _A) * _C, dtype, intervals)
    return _k_as(x * 0.5, dtype, intervals) * 0.5 + 0.5


def _activated(x, activation, dtype, intervals):
    t = _inner(x, activation, dtype, intervals)
    return (x * 0.5 * (t + 1.0) if activation == "gelu" else x * t).to(dtype)


def _slope(x, activation, dtype, intervals):
    t = _inner(x, activation, dtype, intervals)
    if activation == "gelu":
        return (t + 1.0) * 0.5 + x * 0.5 * ((1.0 - t * t) * ((x * x * _A3 + 1.0) * _C))
    return t + x * (t * (1.0 - t))


def _plain_linear(state):
    case, x = state["case"], state["x"]
    if case["activation"]:
        x = _activated(x.float(), case["activation"], x.dtype, case["intervals"])
    x = x.float()
    top = x.abs().amax(1, keepdim=True)
    return {"out": _plain_scaled(state, _codes(x, top), _by(top, 127.0))}


def _plain_product(state):
    return {"out": _plain_scaled(state, state["tokens"].float(), state["token_scale"][:, None])}


def _plain_scaled(state, codes, scale):
    out = torch.matmul(codes, state["weight"].float().t()) * scale * state["weight_scale"]
    if state["bias"] is not None:
        out = out + state["bias"]
    return out.to(_TYPES[state["case"]["out"]])


def _grouped(x):
    """A flat tensor as rows of GROUP values, zeros behind the last."""
    return torch.nn.functional.pad(x, (0, -x.numel() % GROUP)).view(-1, GROUP)


def _checkpoint(x):
    """(codes, scales) of a flat Float32 tensor."""
    rows = _grouped(x)
    top = rows.abs().amax(1, keepdim=True)
    return _codes(rows, top).to(torch.int8).flatten()[:x.numel()].contiguous(), _by(top, 127.0).squeeze(1)


def _restored(codes, scales, dtype):
    """The values that a checkpoint stands for, in Float32."""
    return (_grouped(codes.float()) * scales[:, None]).flatten()[:codes.numel()].to(dtype).float()


def _plain_keep(state):
    case, x, dy = state["case"], state["x"].detach(), state["dy"]
    wide = x.float()
    y = _activated(wide, case["activation"], x.dtype, case["intervals"])
    kept = _restored(*_checkpoint(wide), x.dtype)
    return {"y": y, "dx": (dy.float() * _slope(kept, case["activation"], x.dtype, case["intervals"])).to(x.dtype)}


def _plain_back(state):
    case, dy = state["case"], state["dy"]
    kept = _restored(state["codes"], state["scales"], dy.dtype)
    return {"dx": (dy.float() * _slope(kept, case["activation"], dy.dtype, case["intervals"])).to(dy.dtype),
            "y": _activated(kept, case["activation"], dy.dtype, case["intervals"])}


def _column(value, like, dtype):
    return value[:, None].to(dtype) if torch.is_tensor(value) else torch.full_like(like, value, dtype=dtype)


def _plain_sample(state):
    """In 64 bits from the weights on: a sum of a whole vocabulary decides between neighbours."""
    case, z, u = state["case"], state["logits"].float(), state["uniform"][:, None].double()
    if case["cap"]:
        z = torch.where(z == -math.inf, z, _k(_by(z, case["cap"]), case["intervals"]) * case["cap"])
    temperature, top_p, min_p = (_column(state[n], u, torch.float64) for n in ("temperature", "top_p", "min_p"))
    if not torch.is_tensor(state["temperature"]):       # settings are Float32 numbers
        temperature, top_p, min_p = (t.float().double() for t in (temperature, top_p, min_p))
    top_k = _column(state["top_k"], u, torch.int64)
    vocabulary = z.shape[1]
    ranked, token = z.sort(dim=1, descending=True, stable=True)
    ranked = ranked.double()
    greedy = temperature <= 0
    w = ((ranked - ranked[:, :1]) / torch.where(greedy, torch.ones_like(temperature), temperature)).exp()
    mass = w.cumsum(1)
    before = torch.cat((torch.zeros_like(u), mass[:, :-1]), 1)
    kept = torch.where((top_k <= 0) | (top_k > vocabulary), vocabulary, top_k)
    kept = torch.minimum(kept, (before < top_p * mass.gather(1, kept - 1)).sum(1, keepdim=True))
    kept = torch.minimum(kept, (w >= min_p).sum(1, keepdim=True)).clamp(min=1)
    kept = torch.where(greedy, 1, kept)
    passed = (mass <= u * mass.gather(1, kept - 1)).sum(1, keepdim=True)
    return {"tokens": token.gather(1, torch.minimum(passed, kept - 1)).squeeze(1)}


# -------------------------------------------------------------------------------------------- work

_BYTES = {"bf16": 2, "f32": 4}


def work(case):
    kind, size = case["kind"], _BYTES[case["type"]]
    if kind in ("linear", "product"):
        tokens, inner, outer = case["tokens"], case["inner"], case["outer"]
        each = size * inner if kind == "linear" else inner + 4
        return {"bytes": tokens * each + outer * (inner + 4 + 4 * case["bias"]) + tokens * outer * _BYTES[case["out"]],
                "flops": 2 * tokens * inner * outer}
    if kind in ("keep", "back"):
        # a value and its code, and a scale in 128: y = f(x) writes the code, dx = dy f'(code) (and y, rebuilt) reads it
        kept = 1 + 4 / GROUP
        return {"bytes": int(case["count"] * ((4 * size + 2 * kept) if kind == "keep" else (3 * size + kept))), "flops": 40 * case["count"]}
    return {"bytes": case["rows"] * (case["vocabulary"] * size + 12), "flops": 4 * case["rows"] * case["vocabulary"]}


# ------------------------------------------------------------------------------------------- exact


def _k64(x, intervals):
    """Algorithm 1 on doubles that hold Float32 values: thresholds, index, shift of the 23-bit mantissa and add."""
    lead = 4 if intervals == 64 else 3
    mag = x.abs()
    fraction, exponent = torch.frexp(mag.clamp(0.25, 3.9999997))        # in [0.5, 1)
    mantissa = (fraction * 2 - 1) * 2.0 ** 23
    t = ((exponent.long() + 126) & 3) * 2 ** lead + (mantissa / 2.0 ** (23 - lead)).floor().long()
    E, r, b = (_E64, _R64, _B64) if intervals == 64 else (_E32, _R32, _B32)
    size, shift, offset = (torch.tensor(u, dtype=torch.float64, device=x.device)[t]      # powers of two are the host's: exact
                           for u in ([2.0 ** (e - 127) for e in E], [2.0 ** -e for e in r], [e * 2.0 ** 16 for e in b]))
    out = size * (1.0 + ((mantissa * shift).floor() + offset) * 2.0 ** -23)
    return torch.sign(x) * torch.where(mag < 0.25, mag, torch.where(mag >= 4.0, torch.ones_like(mag), out))


def _inner64(x, case):
    """K at the argument that the definition rounds: it jumps at the ends of its intervals, so the argument is formed with
    the roundings of the definition, one an operation; everything behind it is in 64 bits."""
    x32, bf16 = x.float(), case["type"] == "bf16"
    if case["activation"] == "gelu":
        cube = torch.mul(torch.mul(x32, x32), x32)
        at = torch.mul(torch.add(x32, torch.mul(cube, 0.044715)), 0.7978845608028654)
    else:
        at = torch.mul(x32, 0.5)
    if bf16:
        at = at.bfloat16()
    k = _k64(at.double(), case["intervals"])
    if bf16:        # the mantissa has 7 bits; what is behind them is cut off
        k = (k.float().view(torch.int32) >> 16 << 16).view(torch.float32).double()
    return k


def _value64(x, case):
    k = _inner64(x, case)
    return x * (0.5 + 0.5 * k)


def _slope64(x, case):
    k = _inner64(x, case)
    if case["activation"] == "swish":
        s = 0.5 + 0.5 * k
        return s + x * s * (1 - s)
    return 0.5 * (1 + k) + 0.5 * x * (1 - k ** 2) * _C * (1 + 3 * _A * x ** 2)


def _integers64(x, dim):
    """Integers and scales by the definition's Float32 divisions and products, each rounded from doubles."""
    top = x.abs().amax(dim, keepdim=True)
    inverse = torch.where(top > 0, 127.0 / top, torch.zeros_like(top)).float().double()
    return torch.round((x * inverse).float().double()), _by(top, 127.0).float().double()


def exact(case, seed):
    kind = case["kind"]
    state = prepare(case, seed)
    with torch.no_grad():
        if kind in ("linear", "product"):
            if kind == "linear":
                x = state["x"].double()
                if case["activation"]:
                    x = _value64(x, case).to(_TYPES[case["type"]]).double()
                tokens, scale = _integers64(x, 1)
            else:
                tokens, scale = state["tokens"].double(), state["token_scale"].double()[:, None]
            weight = state["weight"].double() * state["weight_scale"].double()[:, None]
            out = (tokens * scale) @ weight.T
            return {"out": out if state["bias"] is None else out + state["bias"].double()}
        if kind in ("keep", "back"):
            dy = state["dy"].double()
            if kind == "keep":
                x = state["x"].double()
                padded = torch.cat((x, x.new_zeros(-len(x) % GROUP))).unflatten(0, (-1, GROUP))
                codes, scales = _integers64(padded, 1)
            else:
                codes = torch.cat((state["codes"].double(), dy.new_zeros(-len(dy) % GROUP))).unflatten(0, (-1, GROUP))
                scales = state["scales"].double()[:, None]
            kept = (codes * scales).flatten()[:len(dy)].float().to(_TYPES[case["type"]]).double()
            dx = dy * _slope64(kept, case)
            return {"y": _value64(x, case), "dx": dx} if kind == "keep" else {"dx": dx, "y": _value64(kept, case)}
        return {"tokens": torch.tensor([_token64(state, row) for row in range(case["rows"])], device="cuda")}


def _token64(state, row):
    """One row, by its distinct logits: how many tokens share each, and what they weigh together."""
    case = state["case"]

    def setting(name):
        value = state[name]
        return value[row].item() if torch.is_tensor(value) else torch.tensor(value, dtype=torch.float32).item()
    logits = state["logits"][row].float()
    if case["cap"]:
        capped = _k64((_by(logits.double(), case["cap"])).float().double(), case["intervals"]) * case["cap"]
        logits = torch.where(logits == -math.inf, logits.double(), capped).float()
    values, counts = torch.unique(logits + 0.0, return_counts=True)     # + 0.0: one zero
    values, counts = values.flip(0), counts.flip(0)
    temperature = setting("temperature")
    if temperature <= 0:
        return int((logits == values[0]).nonzero()[0])
    each = torch.exp((values.double() - values[0].double()) / temperature)
    up_to = torch.cumsum(each * counts, 0)
    ranks = counts.cumsum(0)

    def mass(count):        # of the first `count` tokens
        at = int(torch.searchsorted(ranks, count))
        return float(up_to[at]) - float(each[at]) * (int(ranks[at]) - count)

    def first(reached):     # the rank of the first token with which the mass satisfies `reached`, from 0
        at = int(torch.nonzero(reached(up_to))[0])
        before = float(up_to[at - 1]) if at else 0.0
        taken = before + float(each[at]) * torch.arange(1, int(counts[at]) + 1, dtype=torch.float64)
        inside = torch.nonzero(reached(taken))
        return int(ranks[at]) - int(counts[at]) + (int(inside[0]) if len(inside) else int(counts[at]) - 1)
    kept = len(logits)
    if 0 < setting("top_k") < kept:
        kept = int(setting("top_k"))
    wanted = setting("top_p") * mass(kept)
    if wanted < float(up_to[-1]):
        kept = min(kept, first(lambda m: m >= wanted) + 1)
    kept = max(1, min(kept, int(counts[each >= setting("min_p")].sum())))
    target = float(state["uniform"][row]) * mass(kept)
    rank = min(first(lambda m: m > target), kept - 1)
    at = int(torch.searchsorted(ranks, rank + 1))
    return int((logits == values[at]).nonzero()[rank - int(ranks[at]) + int(counts[at])])
