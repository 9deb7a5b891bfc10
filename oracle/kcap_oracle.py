"""CPU reference of attention with scores capped through K-TanH, in 64 bits (numpy), and of the cache that goes with it.

Test infrastructure only.  K-TanH itself comes from the C oracle (``ktanh_oracle.ktanh_f32``, ``ktanh64_f32``) on the Float32
rounding of its argument; ``tanh=True`` puts TanH in its place, for which the gradient's formula is the derivative and can be held
against differences.  Every result comes with a bound on how far a computation may be off that rounds where the library does: weights and the
scores' gradients to BFloat16 (2^-8 of a value each: it has eight significant bits), results to BFloat16, and Float32 sums.
"""
from __future__ import annotations

import numpy as np

from . import ktanh_oracle

HALF = 2.0 ** -8     # of a value: what rounding it to BFloat16 may change
F32 = 2.0 ** -24


def k_of(x, intervals=32, lut=None, tanh=False):
    if tanh:
        return np.tanh(x)
    fn = ktanh_oracle.ktanh_f32 if intervals == 32 else ktanh_oracle.ktanh64_f32
    flat = np.ascontiguousarray(x, dtype=np.float32).reshape(-1)
    return fn(flat.view(np.uint32), lut).view(np.float32).astype(np.float64).reshape(x.shape)


def seen(rows, keys, causal, window):
    place = np.arange(rows)[:, None] + (keys - rows)
    key = np.arange(keys)[None, :]
    ok = np.ones((rows, keys), dtype=bool)
    if causal:
        ok &= key <= place
    if window:
        ok &= key > place - window
    return ok


def head(q, k, v, *, cap, scale, causal=True, window=0, intervals=32, lut=None, tanh=False, do=None):
    """One head of one document: q [rows, dim], k and v [keys, dim] as doubles.  A dict of results and of their bounds (`.._off`)."""
    rows, keys, dim = q.shape[0], k.shape[0], q.shape[1]
    ok = seen(rows, keys, causal, window)
    with np.errstate(all="ignore"):
        s = np.where(ok, q @ k.T, 0.0)
    c = scale / cap
    t = k_of(s * (c if tanh else np.float64(np.float32(c))), intervals, lut, tanh)
    y = cap * t
    e = np.where(ok, np.exp(y), 0.0)
    total = e.sum(1)
    some = total > 0
    p = e / np.where(some, total, 1.0)[:, None]
    vs = np.where(np.isfinite(v), v, 0.0)
    o = p @ vs
    for sign in (1, -1):           # an infinite or NaN value reaches the rows that see it
        special = (np.isnan(v) | (v == sign * np.inf)).astype(float)
        if special.any():
            with np.errstate(invalid="ignore"):     # both infinities: NaN
                o = o + np.where(ok.astype(float) @ special > 0, sign * np.inf, 0.0)
    lse = np.where(some, np.log(np.where(some, total, 1.0)), -np.inf)
    # y is off by a few roundings of products up to cap * log2 e: the same share of each weight, and again through the sum
    weight = 2 * 8 * F32 * cap + keys * F32
    # Weights p (1 + d), |d| <= HALF, stand in the numerators and in the sum that divides them: o is off by
    # sum p d (v - o) / sum p (1 + d), and sum p |v - o| is no more than the root of sum p (v - o)^2.
    mean = p @ vs
    spread = np.sqrt(np.maximum(p @ (vs * vs) - mean * mean, 0.0) + 1e-15 * (p @ (vs * vs)))
    o_off = HALF / (1 - HALF) * spread + weight * (p @ np.abs(vs))
    o_off = o_off + HALF * (np.abs(o) + o_off) + 1e-30
    out = {"o": o, "lse": lse, "o_off": o_off, "lse_off": weight + 4 * F32 * np.abs(np.where(some, lse, 0.0))}
    if do is None:
        return out
    dp = do @ v.T
    slope = 1.0 - t * t
    delta = (do * o).sum(1, keepdims=True)
    ds = p * (dp - delta) * slope
    out.update(dq=scale * ds @ k, dk=scale * ds.T @ q, dv=p.T @ do)
    # delta is formed from the rounded output
    delta_off = (np.abs(do) * o_off).sum(1, keepdims=True) + dim * F32 * (np.abs(do) * np.abs(o)).sum(1, keepdims=True)
    dp_off = dim * F32 * (np.abs(do) @ np.abs(v).T)
    ds_off = HALF * np.abs(ds) + p * np.abs(slope) * (delta_off + dp_off) + (weight + 8 * F32) * p * (np.abs(dp) + np.abs(delta))
    sums = (rows + keys) * F32
    for name, off, with_ in (("dq", ds_off, k), ("dk", ds_off.T, q)):
        share = ds if name == "dq" else ds.T
        out[name + "_off"] = abs(scale) * (off @ np.abs(with_) + sums * (np.abs(share) @ np.abs(with_))) + HALF * np.abs(out[name]) + 1e-30
    out["dv_off"] = (HALF + weight + sums) * (p.T @ np.abs(do)) + HALF * np.abs(out["dv"]) + 1e-30
    return out


def attention(q, k, v, q_offsets, k_offsets, do=None, **options):
    """All heads and documents: q [rows, heads, dim], k and v [keys, kv_heads, dim] as doubles."""
    heads, kv_heads = q.shape[1], k.shape[1]
    group = heads // kv_heads
    made = {"o": np.zeros(q.shape), "lse": np.full((heads, q.shape[0]), -np.inf)}
    made.update(o_off=np.zeros(q.shape), lse_off=np.zeros(made["lse"].shape))
    if do is not None:
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            made[name], made[name + "_off"] = np.zeros(like.shape), np.zeros(like.shape)
    for d in range(len(q_offsets) - 1):
        rows, keys = slice(q_offsets[d], q_offsets[d + 1]), slice(k_offsets[d], k_offsets[d + 1])
        for h in range(heads):
            kv = h // group
            one = head(q[rows, h], k[keys, kv], v[keys, kv], do=None if do is None else do[rows, h], **options)
            for name in ("o", "o_off"):
                made[name][rows, h] = one[name]
            for name in ("lse", "lse_off"):
                made[name][h, rows] = one[name]
            if do is not None:
                for name in ("dq", "dq_off"):
                    made[name][rows, h] = one[name]
                for name in ("dk", "dk_off", "dv", "dv_off"):   # shared heads add up
                    made[name][keys, kv] += one[name]
    return made


def gather(cache, pages, length):
    """[length, kv_heads, dim] of one sequence from a cache [pages, page size, kv_heads, dim]."""
    page = cache.shape[1]
    return cache[pages[:-(-length // page)]].reshape(-1, *cache.shape[2:])[:length]


def turned(x, cos, sin, interleaved):
    """x [heads, dim] rotated by cos, sin [angles]."""
    n = len(cos)
    out = x.copy()
    a, b = (x[:, 0:2 * n:2], x[:, 1:2 * n:2]) if interleaved else (x[:, :n], x[:, n:2 * n])
    first, second = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        out[:, 0:2 * n:2], out[:, 1:2 * n:2] = first, second
    else:
        out[:, :n], out[:, n:2 * n] = first, second
    return out
