"""Capped attention on ordinary BFloat16 inputs, whose q.k rounds in Float32: K-TanH jumps at the ends of its intervals, and a score near one may
fall on either side.

The bound adds to the reference's what such scores may change.  The scores of any order of summation lie within 2 dim 2^-24 sum |q||k| of the exact
ones (bfloat16 products are exact in Float32; twice, for sums that cut off instead of rounding), the arguments x of K within `away`.  There K is
off by D = max |K(x +- away) - K(x)|: both sides of a jump if one is that near, and the slope of the line elsewhere.  A weight p then lies between
p e^(-cap D) / sum p e^(cap D) and p e^(cap D) / sum p e^(-cap D), and outputs and gradients follow from their formulas term by term."""
import numpy as np
import pytest

from oracle import kcap_oracle
from test_gpu_cap_attention import _bf16, _near, _offsets, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _extra(q, k, v, do, *, cap, scale, causal=True, window=0, intervals=32):
    """What scores off by their rounding may change in one head: of o, lse, dq, dk, dv; and how many of the seen scores are near a jump."""
    rows, keys, dim = len(q), len(k), q.shape[1]
    ok = kcap_oracle.seen(rows, keys, causal, window)
    x = q @ k.T * np.float64(np.float32(scale / cap))
    away = 2.0 ** -24 * (2 * dim * (np.abs(q) @ np.abs(k).T) * abs(scale / cap) + 4 * np.abs(x))
    t = kcap_oracle.k_of(x, intervals)
    off = np.where(ok, np.maximum(np.abs(kcap_oracle.k_of(x + away, intervals) - t), np.abs(kcap_oracle.k_of(x - away, intervals) - t)), 0.0)
    p = np.where(ok, np.exp(cap * t), 0.0)
    total = p.sum(1, keepdims=True)
    p = p / np.where(total > 0, total, 1.0)
    high, low = (p * np.exp(cap * off)), (p * np.exp(-cap * off))
    most, least = high.sum(1, keepdims=True), low.sum(1, keepdims=True)
    moved = np.maximum(high / np.where(least > 0, least, 1.0) - p, p - low / np.where(most > 0, most, 1.0))
    o = p @ v
    o_off = np.stack([(moved * np.abs(v[None, :, d] - o[:, None, d])).sum(1) for d in range(dim)], 1)
    with np.errstate(divide="ignore"):
        lse_off = np.where(least[:, 0] > 0, np.maximum(np.log(most[:, 0]), -np.log(least[:, 0])), 0.0)
    out = {"o": o_off, "lse": lse_off, "near": int((ok & (off > 4 * away)).sum())}
    if do is not None:
        dp, slope = do @ v.T, 1.0 - t * t
        delta = (do * o).sum(1, keepdims=True)
        delta_off = (np.abs(do) * o_off).sum(1, keepdims=True)
        ds_off = moved * np.abs((dp - delta) * slope) + (p + moved) * (delta_off * np.abs(slope) + (np.abs(dp - delta) + delta_off) * (2 * np.abs(t) + off) * off)
        out.update(dq=abs(scale) * ds_off @ np.abs(k), dk=abs(scale) * ds_off.T @ np.abs(q), dv=moved.T @ np.abs(do))
    return out


def _allowed(want, wide, do, q_at, k_at, **options):
    """The reference's bounds with _extra of every document and head, and the scores near a jump."""
    q, k, v = wide
    group, near = q.shape[1] // k.shape[1], 0
    off = {n: want[n + "_off"].copy() for n in ("o", "lse", "dq", "dk", "dv") if n in want}
    for d in range(len(q_at) - 1):
        r, c = slice(q_at[d], q_at[d + 1]), slice(k_at[d], k_at[d + 1])
        for h in range(q.shape[1]):
            one = _extra(q[r, h], k[c, h // group], v[c, h // group], None if do is None else do[r, h], **options)
            near += one["near"]
            off["o"][r, h] += one["o"] * (1 + 2.0 ** -8)        # and its rounding
            off["lse"][h, r] += one["lse"]
            if do is not None:
                off["dq"][r, h] += one["dq"] * (1 + 2.0 ** -6)  # of P, dS and the result
                off["dk"][c, h // group] += one["dk"] * (1 + 2.0 ** -6)
                off["dv"][c, h // group] += one["dv"] * (1 + 2.0 ** -6)
    return off, near


def _ordinary(torch, seed, *shapes):
    rng = np.random.default_rng(seed)
    tensors = [_bf16(torch, rng.standard_normal(s) * w) for s, w in shapes]
    return tensors, [t.double().cpu().numpy() for t in tensors]


@pytest.mark.parametrize("options", [dict(cap=50.0, causal=True), dict(cap=30.0, causal=False), dict(cap=20.0, causal=True, window=50)])
@pytest.mark.parametrize("heads,kv_heads,dim,intervals", [(4, 2, 128, 32), (4, 2, 64, 64), (192, 2, 64, 32)])
def test_documents_and_gradients(gpu, options, heads, kv_heads, dim, intervals):  # noqa: F811
    binding, autograd, torch = gpu
    lengths = [130, 1, 77]
    rows = sum(lengths)
    (q, k, v, do), wide = _ordinary(torch, 60, ((rows, heads, dim), 10.0), ((rows, kv_heads, dim), 1.0), ((rows, kv_heads, dim), 1.0), ((rows, heads, dim), 1.0))
    at, at_np = _offsets(torch, lengths)
    options = dict(options, scale=dim ** -0.5)
    attend = binding.kcap_attention if intervals == 32 else binding.kcap_attention64
    o, lse = attend(q, k, v, at, **options)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    made = autograd.kcap_attention(*leaves, at, intervals=intervals, **options)
    grads = torch.autograd.grad(made, leaves, do)
    assert torch.equal(made.detach(), o)
    want = kcap_oracle.attention(*wide[:3], at_np, at_np, do=wide[3], intervals=intervals, **options)
    off, near = _allowed(want, wide[:3], wide[3], at_np, at_np, intervals=intervals, **options)
    assert near > 0
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        _near(got, want[name], off[name], name)
        # jumps are rare: most of the bound is the roundings' (log-sums have next to none of those)
        assert name == "lse" or np.median(off[name]) <= 1.5 * np.median(want[name + "_off"]), name


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (3, 3, 64)])
def test_over_pages(gpu, heads, kv_heads, dim):  # noqa: F811
    binding, _, torch = gpu
    lengths = [700, 33, 1]
    most = -(-max(lengths) // 16)
    (q, k, v), wide = _ordinary(torch, 61, ((len(lengths), heads, dim), 10.0), ((len(lengths), most * 16, kv_heads, dim), 1.0), ((len(lengths), most * 16, kv_heads, dim), 1.0))
    pages = torch.arange(len(lengths) * most, dtype=torch.int32, device="cuda").view(len(lengths), most)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    one = torch.arange(len(lengths) + 1, dtype=torch.int32, device="cuda")
    options = dict(cap=50.0, scale=dim ** -0.5)
    caches = [t.view(-1, 16, kv_heads, dim) for t in (k, v)]
    single = binding.kcap_attention_paged(q, *caches, pages, n, **options)
    pieces = binding.kcap_attention_paged(q, *caches, pages, n, one, **options)
    for s, keys in enumerate(lengths):
        mine = [wide[0][s:s + 1], wide[1][s, :keys], wide[2][s, :keys]]
        want = kcap_oracle.attention(*mine, [0, 1], [0, keys], **options)
        off, _ = _allowed(want, mine, None, [0, 1], [0, keys], **options)
        _near(single[s:s + 1], want["o"], off["o"], f"single, sequence {s}")
        _near(pieces[s:s + 1], want["o"], off["o"], f"pieces, sequence {s}")
