"""Attention with scores capped through K-TanH against a 64-bit reference: packed documents, shared heads, masks that leave
rows empty, values that are not finite behind masks, strides, streams, the paged cache and the appending to it.

q and k are multiples of 1/8 below 8, so that every q.k is exact in Float32 and both sides see the same interval of K-TanH's table;
the bounds are the reference's own (what rounding weights, scores' gradients and results to BFloat16 may change)."""
import numpy as np
import pytest

from oracle import kcap_oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu(oracle):
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1909_07729_amd import autograd, binding
    binding.load_library()
    torch.cuda.set_device(0)
    return binding, autograd, torch


def _grid(rng, shape, spread):
    return np.clip(np.round(rng.standard_normal(shape) * spread * 8), -63, 63) / 8


def _bf16(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().bfloat16()


def _inputs(torch, seed, q_rows, k_rows, heads, kv_heads, dim, spread=2.0):
    """(device tensors q, k, v), (the same as doubles)"""
    rng = np.random.default_rng(seed)
    arrays = [_grid(rng, (q_rows, heads, dim), spread), _grid(rng, (k_rows, kv_heads, dim), spread), rng.standard_normal((k_rows, kv_heads, dim))]
    tensors = [_bf16(torch, a) for a in arrays]
    return tensors, [t.float().cpu().numpy().astype(np.float64) for t in tensors]


def _offsets(torch, lengths):
    at = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    return torch.from_numpy(at).cuda(), at


def _near(got, want, off, what):
    got = got.float().cpu().numpy().astype(np.float64) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{what}: infinities elsewhere"
    far = np.abs(got[fine] - want[fine])
    assert (far <= off[fine]).all(), f"{what}: {(far / np.maximum(off[fine], 1e-30)).max():.2f} of the bound"


# (query lengths, key lengths or None for the same)
DOCS = {
    "one token": ([1], None),
    "one of each size around a tile": ([63, 64, 65, 1, 0, 127, 128, 129, 2], None),
    "one long": ([401], None),
    "empty documents": ([0, 5, 0, 0, 70, 0], None),
    "fewer queries than keys": ([3, 1, 60, 130], [200, 64, 61, 131]),
    "more queries than keys": ([40, 130, 7, 4], [5, 64, 0, 3]),
}
MASKS = {"causal": dict(causal=True), "all": dict(causal=False), "window": dict(causal=True, window=37),
         "window of one": dict(causal=True, window=1), "window, later keys too": dict(causal=False, window=70),
         "window beyond 32 bits": dict(causal=True, window=1 << 40)}
HEADS = [(1, 1, 64), (4, 2, 128), (5, 1, 64), (3, 3, 128)]


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("docs", DOCS)
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_documents(gpu, docs, mask, heads, kv_heads, dim):
    binding, _, torch = gpu
    q_lengths, k_lengths = DOCS[docs]
    k_lengths = q_lengths if k_lengths is None else k_lengths
    (q, k, v), wide = _inputs(torch, 1, sum(q_lengths), sum(k_lengths), heads, kv_heads, dim)
    (q_at, q_np), (k_at, k_np) = _offsets(torch, q_lengths), _offsets(torch, k_lengths)
    options = dict(cap=32.0, scale=dim ** -0.5, **MASKS[mask])
    o, lse = binding.kcap_attention(q, k, v, q_at, k_at, **options)
    want = kcap_oracle.attention(*wide, q_np, k_np, **options)
    _near(o, want["o"], want["o_off"], "o")
    _near(lse, want["lse"], want["lse_off"], "lse")
    empty = np.isinf(want["lse"])
    assert not o.float().cpu().numpy().transpose(1, 0, 2)[empty].any()


@pytest.mark.parametrize("intervals", [32, 64])
@pytest.mark.parametrize("cap,spread", [(0.5, 2.0), (20.0, 3.0), (50.0, 3.0), (64.0, 4.0), (64.0, 0.2)])
def test_caps_and_tables(gpu, cap, spread, intervals):
    """From saturated scores (cap 0.5) to ones that never leave the identity, with the default and a caller's tables."""
    binding, _, torch = gpu
    (q, k, v), wide = _inputs(torch, 2, 150, 150, 2, 1, 128, spread)
    at, at_np = _offsets(torch, [150])
    entry = binding.kcap_attention if intervals == 32 else binding.kcap_attention64
    tables = [(None, None)]
    from oracle import ktanh_oracle
    if intervals == 32:
        tables.append((binding.ktanh_fit_lut_bmin0(), ktanh_oracle.fit_lut_bmin0()))
    else:
        rows = binding.ktanh_fit_lut64().as_tuples()
        rows[20] = (125, 1, 3)
        tables.append((binding.KtanhLut64.from_tuples(rows), ktanh_oracle.OracleLut64.from_tuples(rows)))
    for lut, oracle_lut in tables:
        options = dict(cap=cap, scale=128 ** -0.5)
        o, lse = entry(q, k, v, at, lut=lut, **options)
        want = kcap_oracle.attention(*wide, at_np, at_np, intervals=intervals, lut=oracle_lut, **options)
        _near(o, want["o"], want["o_off"], "o")
        _near(lse, want["lse"], want["lse_off"], "lse")


@pytest.mark.parametrize("heads", [2, 512])
@pytest.mark.parametrize("cap,keys", [(64.0, 3000), (64.0, 60), (50.0, 1000)])
def test_values_up_to_what_the_sums_hold(gpu, cap, keys, heads):
    """Scores that are all at the cap and values up to 3e38 / (keys e^cap), over documents and over pages: no sum leaves Float32."""
    binding, _, torch = gpu
    largest = 3e38 / (keys * np.exp(cap))
    k64, v64 = np.full((keys, 1, 64), 8.0), np.full((keys, 1, 64), largest)
    v64[:, :, 1::2] *= np.random.default_rng(51).uniform(-1.0, 1.0, (keys, 1, 32))
    k, v = _bf16(torch, k64), _bf16(torch, v64)
    v = torch.where(v.abs() > largest, v * (1 - 2.0 ** -7), v)        # rounding to BFloat16 may have gone beyond
    v64, q64 = v.double().cpu().numpy(), np.full((2, heads, 64), 7.0)
    options = dict(cap=cap, scale=1.0)                           # x is 56 and more
    want = kcap_oracle.attention(q64[:, :1], k64, v64, [0, 2], [0, keys], **options)
    want, off = (np.broadcast_to(want[n], q64.shape) for n in ("o", "o_off"))
    assert np.isfinite(want).all()
    q, at, at_k = _bf16(torch, q64), _offsets(torch, [2])[0], _offsets(torch, [keys])[0]
    _near(binding.kcap_attention(q, k, v, at, at_k, **options)[0], want, off, "documents")
    pages = -(-keys // 16)
    k_cache, v_cache = (torch.cat([t, t.new_zeros((pages * 16 - keys, 1, 64))]).view(pages, 16, 1, 64) for t in (k, v))
    table, n = torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.tensor([keys], dtype=torch.int32, device="cuda")
    _near(binding.kcap_attention_paged(q, k_cache, v_cache, table, n, at, **options), want, off, "pieces")
    _near(binding.kcap_attention_paged(q[1:], k_cache, v_cache, table, n, **options), want[1:], off[1:], "single")


@pytest.mark.parametrize("mask", ["causal", "window", "all"])
def test_what_is_not_seen_does_not_reach_a_row(gpu, mask):
    """NaN and infinities in keys and values: of other documents, later than the query, before its window, and in rows of no document."""
    binding, _, torch = gpu
    (q, k, v), (q64, k64, v64) = _inputs(torch, 3, 300, 300, 2, 1, 64)
    at, at_np = _offsets(torch, [90, 140])          # the last 70 rows belong to nobody
    rng = np.random.default_rng(4)
    for value in (np.nan, np.inf, -np.inf):
        for j in rng.integers(0, 300, 4):
            v64[j, 0, rng.integers(0, 64, 3)] = value
    for j in (250,) if mask == "all" else (80, 229, 250):
        k64[j, 0, 5] = np.nan
    k, v = _bf16(torch, k64), _bf16(torch, v64)
    v64 = v.float().cpu().numpy().astype(np.float64)
    options = dict(cap=32.0, scale=0.125, **MASKS[mask])
    o, _ = binding.kcap_attention(q, k, v, at, **options)
    want = kcap_oracle.attention(q64, k64, v64, at_np, at_np, **options)["o"]
    # rows that see a NaN key are NaN
    for d, (a, b) in enumerate(zip(at_np[:-1], at_np[1:])):
        ok = kcap_oracle.seen(b - a, b - a, options.get("causal", True), options.get("window", 0))
        bad = ok @ np.isnan(k64[a:b, 0]).any(1)
        want[a:b][bad] = np.nan
    got = o.float().cpu().numpy()[:230]
    assert np.isfinite(want[:230]).any() and not np.isfinite(want[:230]).all()
    assert np.array_equal(np.isnan(got), np.isnan(want[:230]))
    fine = ~np.isnan(got)
    assert np.array_equal(np.isinf(got)[fine], np.isinf(want[:230])[fine])


def test_strided_tensors_and_given_outputs(gpu):
    """q, k and v as views of one fused tensor, heads before rows, results in the caller's memory, zeros in rows of no document."""
    binding, _, torch = gpu
    (q, k, v), wide = _inputs(torch, 5, 200, 200, 4, 2, 64)
    fused = torch.cat([q, k, v], 1).contiguous()
    views = fused[:, :4], fused[:, 4:6], fused[:, 6:]
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    at, at_np = _offsets(torch, [31, 150])
    options = dict(cap=50.0, scale=0.125)
    want = kcap_oracle.attention(*wide, at_np, at_np, **options)
    first = None
    for tensors in ((q, k, v), views, turned):
        out = torch.full((200, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((4, 200), 7.0, device="cuda")
        o, sums = binding.kcap_attention(*tensors, at, out=out, lse=lse, **options)
        assert o is out and sums is lse
        _near(o[:181], want["o"][:181], want["o_off"][:181], "o")
        assert (o[181:] == 0).all() and (lse[:, 181:] == -float("inf")).all()
        first = o.clone() if first is None else first
        assert torch.equal(o, first)


def test_offsets_out_of_range_read_nothing_out_of_bounds(gpu):
    binding, _, torch = gpu
    (q, k, v), wide = _inputs(torch, 6, 100, 100, 2, 2, 64)
    options = dict(cap=50.0, scale=0.125, causal=False)
    wrong = torch.tensor([-5, 60, 1000], dtype=torch.int32, device="cuda")
    right = torch.tensor([0, 60, 100], dtype=torch.int32, device="cuda")
    a, b = (binding.kcap_attention(q, k, v, at, **options)[0] for at in (wrong, right))
    assert torch.equal(a, b)


def test_many_documents(gpu):
    """More documents than a wavefront looks at in one step."""
    binding, _, torch = gpu
    rng = np.random.default_rng(7)
    lengths = rng.integers(0, 9, 300)
    (q, k, v), wide = _inputs(torch, 8, lengths.sum(), lengths.sum(), 2, 1, 64)
    at, at_np = _offsets(torch, lengths)
    options = dict(cap=50.0, scale=0.125)
    o, lse = binding.kcap_attention(q, k, v, at, **options)
    want = kcap_oracle.attention(*wide, at_np, at_np, **options)
    _near(o, want["o"], want["o_off"], "o")
    _near(lse, want["lse"], want["lse_off"], "lse")


@pytest.mark.parametrize("mask", ["causal", "all", "window"])
@pytest.mark.parametrize("docs", [2, 64, 65, 200])
def test_numbers_of_documents_behind_rows_of_none(gpu, docs, mask):
    """Up to 64 documents blocks go by work, beyond by rows; 300 rows of no document before the first and behind the last."""
    rng = np.random.default_rng(40)
    lengths = rng.integers(0, 20, docs)
    lengths[docs // 2] = 290
    got, want = _grads(gpu, 41, lengths.tolist(), lengths.tolist(), 2, 1, 64, lead=300, cap=50.0, scale=0.125, **MASKS[mask])
    for name, t in got.items():
        _near(t, want[name], want[name + "_off"], name)


def test_on_another_stream_and_in_a_graph(gpu):
    binding, _, torch = gpu
    (q, k, v), _ = _inputs(torch, 9, 500, 500, 2, 1, 128)
    at, _ = _offsets(torch, [500])
    want, _ = binding.kcap_attention(q, k, v, at, cap=50.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = binding.kcap_attention(q, k, v, at, cap=50.0, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, _ = binding.kcap_attention(q, k, v, at, cap=50.0)
    for scale in (1.0, 0.5, 2.0):
        v.copy_(v * scale)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, binding.kcap_attention(q, k, v, at, cap=50.0)[0])


# ---------------------------------------------------------------------------------------- gradients


def _grads(gpu, seed, q_lengths, k_lengths, heads, kv_heads, dim, spread=2.0, intervals=32, lead=0, **options):
    """Gradients through autograd and their reference, with `lead` rows of no document before and behind."""
    binding, autograd, torch = gpu
    q_rows, k_rows = sum(q_lengths) + 2 * lead, sum(k_lengths) + 2 * lead
    tensors, wide = _inputs(torch, seed, q_rows, k_rows, heads, kv_heads, dim, spread)
    do = _bf16(torch, np.random.default_rng(seed + 1).standard_normal((q_rows, heads, dim)))
    (q_at, q_np), (k_at, k_np) = _offsets(torch, [lead] + list(q_lengths)), _offsets(torch, [lead] + list(k_lengths))
    (q_at, q_np), (k_at, k_np) = (q_at[1:], q_np[1:]), (k_at[1:], k_np[1:])
    leaves = [t.clone().requires_grad_() for t in tensors]
    o = autograd.kcap_attention(*leaves, q_at, k_at, intervals=intervals, **options)
    got = {"o": o.detach(), **dict(zip(("dq", "dk", "dv"), torch.autograd.grad(o, leaves, do)))}
    want = kcap_oracle.attention(*wide, q_np, k_np, do=do.float().cpu().numpy().astype(np.float64), intervals=intervals, **options)
    return got, want


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("docs", DOCS)
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_gradients(gpu, docs, mask, heads, kv_heads, dim):
    q_lengths, k_lengths = DOCS[docs]
    got, want = _grads(gpu, 20, q_lengths, q_lengths if k_lengths is None else k_lengths, heads, kv_heads, dim, lead=3, cap=32.0,
                       scale=dim ** -0.5, **MASKS[mask])
    for name, t in got.items():
        _near(t, want[name], want[name + "_off"], name)


@pytest.mark.parametrize("intervals", [32, 64])
@pytest.mark.parametrize("cap,spread", [(0.5, 2.0), (20.0, 3.0), (50.0, 0.5), (64.0, 4.0)])
def test_gradients_of_caps_and_tables(gpu, cap, spread, intervals):
    got, want = _grads(gpu, 21, [150, 30], [150, 30], 6, 2, 128, spread, intervals, cap=cap, scale=128 ** -0.5)
    for name, t in got.items():
        _near(t, want[name], want[name + "_off"], name)


def _many_heads(docs, kv_heads):
    """Query heads, a multiple of kv_heads, that make 512 blocks of 128 rows or more of the documents."""
    lengths = DOCS[docs][0]
    return -(-512 // (kv_heads * (min(sum(lengths), sum(DOCS[docs][1] or lengths)) // 128 + len(lengths)))) * kv_heads


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("docs", DOCS)
@pytest.mark.parametrize("kv_heads,dim", [(8, 64), (3, 128)])
def test_blocks_of_128_rows(gpu, docs, mask, kv_heads, dim):
    """Many heads: a wavefront goes over all tiles of its 32 rows, where few heads let four share them."""
    heads = _many_heads(docs, kv_heads)
    test_documents(gpu, docs, mask, heads, kv_heads, dim)
    test_gradients(gpu, docs, mask, heads, kv_heads, dim)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_shared_tiles_of_ragged_documents(gpu, mask, heads, kv_heads, dim):
    """Few heads and long enough documents that the four wavefronts of a block share its tiles, with ones of every size around a tile among them."""
    lengths = [65, 0, 1, 127, 700, 33, 128]
    got, want = _grads(gpu, 52, lengths, lengths, heads, kv_heads, dim, lead=3, cap=32.0, scale=dim ** -0.5, **MASKS[mask])
    for name, t in got.items():
        _near(t, want[name], want[name + "_off"], name)


@pytest.mark.parametrize("mask", ["causal", "window"])
def test_what_is_not_seen_does_not_reach_a_row_of_many_heads(gpu, mask):
    binding, _, torch = gpu
    (q, k, v), (q64, k64, v64) = _inputs(torch, 3, 300, 300, 2, 1, 64)
    at, at_np = _offsets(torch, [90, 140])
    for j, value in ((20, np.nan), (85, np.inf), (100, -np.inf), (228, np.nan), (250, np.inf)):
        v64[j, 0, 3:70:20] = value
    k64[229, 0, 5] = k64[250, 0, 5] = np.nan
    options = dict(cap=32.0, scale=0.125, **MASKS[mask])
    o, _ = binding.kcap_attention(q.repeat(1, 128, 1), _bf16(torch, k64), _bf16(torch, v64), at, **options)
    want = kcap_oracle.attention(q64, np.nan_to_num(k64), v64, at_np, at_np, **options)["o"]
    want[229] = np.nan      # the only row that sees the NaN key
    off = kcap_oracle.attention(q64, np.nan_to_num(k64), np.where(np.isfinite(v64), v64, 0.0), at_np, at_np, **options)["o_off"]
    got = o.float().cpu().numpy()
    for head in range(0, 256, 51):
        _near(got[:230, head], want[:230, head % 2], off[:230, head % 2], f"head {head}")


def test_gradients_with_many_blocks_and_with_few_are_the_same(gpu):
    """Enough keys that one block sums all heads of a group, against the same documents in calls of their own, where four wavefronts
    share the tiles of 32 rows."""
    binding, _, torch = gpu
    docs, n = 520, 130
    (q, k, v), _ = _inputs(torch, 22, docs * n, docs * n, 4, 2, 64)
    do = _bf16(torch, np.random.default_rng(23).standard_normal((docs * n, 4, 64)))
    at = torch.arange(0, docs * n + 1, n, dtype=torch.int32, device="cuda")
    o, lse = binding.kcap_attention(q, k, v, at, cap=50.0)
    whole = binding.kcap_attention_backward(do, q, k, v, o, lse, at, cap=50.0)
    one = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    for d in (0, 7, docs - 1):
        rows = slice(d * n, (d + 1) * n)
        parts = binding.kcap_attention_backward(do[rows], q[rows], k[rows], v[rows], o[rows], lse[:, rows].contiguous(), one, cap=50.0)
        for a, b in zip(whole, parts):                  # sums of Float32 in another order, rounded
            assert torch.allclose(a[rows].float(), b.float(), rtol=2 ** -7, atol=2 ** -12)


@pytest.mark.parametrize("heads,kv_heads,dim,q_rows,causal", [(16, 8, 64, 512, True), (16, 1, 128, 512, True), (32, 2, 128, 1024, False),
                                                              (4, 2, 64, 60, True), (3, 1, 128, 60, True)])
def test_gradients_of_keys_that_no_query_sees(gpu, heads, kv_heads, dim, q_rows, causal):
    """Whole blocks of keys without a query, of a document that has none and before the window of one that has few: in blocks of 128 keys,
    with the shared heads in parts (many queries) and in one block (few), their gradients are exactly zero."""
    binding, _, torch = gpu
    keys = 2048
    (q, k, v), _ = _inputs(torch, 46, q_rows, 2 * keys, heads, kv_heads, dim)
    do = _bf16(torch, np.random.default_rng(47).standard_normal((q_rows, heads, dim)))
    (q_at, _), (k_at, _) = _offsets(torch, [q_rows, 0]), _offsets(torch, [keys, keys])
    for window, seen_from in ((0, 0), (64, keys - q_rows - 63)):
        options = dict(cap=50.0, window=window, causal=causal)
        o, lse = binding.kcap_attention(q, k, v, q_at, k_at, **options)
        outs = [torch.full_like(t, 7.0) for t in (q, k, v)]
        binding.kcap_attention_backward(do, q, k, v, o, lse, q_at, k_at, dq=outs[0], dk=outs[1], dv=outs[2], **options)
        for t in outs[1:]:
            assert not t[:seen_from].any() and not t[keys:].any() and t[seen_from:keys].any()


def test_gradients_repeat_and_take_strides(gpu):
    binding, _, torch = gpu
    (q, k, v), _ = _inputs(torch, 24, 400, 400, 4, 2, 64)
    do = _bf16(torch, np.random.default_rng(25).standard_normal((400, 4, 64)))
    at, _ = _offsets(torch, [99, 301])
    options = dict(cap=50.0, scale=0.125, causal=True, window=0)
    o, lse = binding.kcap_attention(q, k, v, at, **options)
    first = binding.kcap_attention_backward(do, q, k, v, o, lse, at, **options)
    fused = torch.cat([q, k, v, do], 1)
    outs = [torch.empty_like(t) for t in first]
    again = binding.kcap_attention_backward(fused[:, 8:], fused[:, :4], fused[:, 4:6], fused[:, 6:8], o, lse, at, dq=outs[0], dk=outs[1],
                                            dv=outs[2], **options)
    for a, b, c in zip(first, again, outs):
        assert b is c and torch.equal(a, b)


def test_gradient_of_a_sum_and_of_shared_inputs(gpu):
    """An expanded incoming gradient, and k and v that are one tensor: their gradients add up."""
    binding, autograd, torch = gpu
    (q, k, _), _ = _inputs(torch, 26, 70, 70, 2, 1, 64)
    at, _ = _offsets(torch, [70])
    q.requires_grad_()
    k.requires_grad_()
    o = autograd.kcap_attention(q, k, k, at, cap=50.0)
    dq, dk = torch.autograd.grad(o.sum(), (q, k))
    rest = torch.empty_like(q)
    o, lse = binding.kcap_attention(q.detach(), k.detach(), k.detach(), at, cap=50.0, rest=rest)
    want = binding.kcap_attention_backward(torch.ones_like(q), q.detach(), k.detach(), k.detach(), o, lse, at, cap=50.0, rest=rest)
    assert torch.equal(dq, want[0]) and torch.equal(dk, want[1] + want[2])


@pytest.mark.parametrize("lut", [False, True])
def test_gradient_with_strides_that_the_kernels_do_not_take(gpu, lut):
    """An incoming gradient heads first, its heads 2^24 elements apart: nothing that the caller of autograd chose."""
    binding, autograd, torch = gpu
    (q, k, v), _ = _inputs(torch, 53, 40, 40, 2, 1, 64)
    at, _ = _offsets(torch, [40])
    far = torch.zeros((1 << 24) + 40 * 64, dtype=torch.bfloat16, device="cuda").as_strided((40, 2, 64), (64, 1 << 24, 1))
    far.copy_(_bf16(torch, np.random.default_rng(54).standard_normal((40, 2, 64))))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    o = autograd.kcap_attention(*leaves, at, cap=50.0, lut=binding.ktanh_default_lut() if lut else None)     # a caller's table takes the Python code
    got = torch.autograd.grad(o, leaves, far, retain_graph=True)
    for a, b in zip(got, torch.autograd.grad(o, leaves, far.contiguous())):
        assert torch.equal(a, b)


def test_what_rounding_dropped(gpu):
    """o and its rest together are the output to sixteen bits; with it the gradients of a peaked head are at least as near."""
    binding, _, torch = gpu
    (q, k, v), wide = _inputs(torch, 29, 200, 200, 2, 1, 128, 2.4)
    do = _bf16(torch, np.random.default_rng(30).standard_normal((200, 2, 128)))
    at, at_np = _offsets(torch, [200])
    options = dict(cap=50.0, scale=128 ** -0.5)
    rest = torch.empty_like(q)
    o, lse = binding.kcap_attention(q, k, v, at, rest=rest, **options)
    plain = binding.kcap_attention(q, k, v, at, **options)
    assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1])
    assert (rest.float().abs() <= 2 ** -8 * o.float().abs()).all() and rest.any()       # half a step of o, itself rounded
    want = kcap_oracle.attention(*wide, at_np, at_np, do=do.float().cpu().numpy().astype(np.float64), **options)

    def off(**more):
        got = binding.kcap_attention_backward(do, q, k, v, o, lse, at, **more, **options)
        return [np.linalg.norm(t.double().cpu().numpy() - want[n]) / np.linalg.norm(want[n]) for n, t in zip(("dq", "dk", "dv"), got)]
    with_rest, without = off(rest=rest), off()
    assert all(a <= b for a, b in zip(with_rest, without)) and max(with_rest) < 4e-3, (with_rest, without)


def test_gradients_against_differences(gpu):
    """Where no score leaves the identity of K-TanH the gradient is that of softmax attention with the slope 1 - x^2: the loss along a
    direction, stepped by 2^-4 of it, differs from the gradient's share by the rounding of q, k and v and the third derivative."""
    binding, autograd, torch = gpu
    (q, k, v), wide = _inputs(torch, 27, 60, 60, 2, 1, 64, 0.5)
    at, at_np = _offsets(torch, [60])
    rng = np.random.default_rng(28)
    do = rng.standard_normal((60, 2, 64))
    leaves = [t.requires_grad_() for t in (q, k, v)]
    o = autograd.kcap_attention(*leaves, at, cap=64.0, scale=0.125)
    grads = torch.autograd.grad(o, leaves, _bf16(torch, do))
    do = _bf16(torch, do).double().cpu().numpy()
    for i in range(3):
        step = rng.integers(-1, 2, wide[i].shape) / 16
        losses = []
        for sign in (1, -1):
            moved = [w + sign * step if j == i else w for j, w in enumerate(wide)]
            losses.append((kcap_oracle.attention(*moved, at_np, at_np, cap=64.0, scale=0.125)["o"] * do).sum())
        along = float((grads[i].double().cpu().numpy() * step).sum())
        # K's slope is 1 below 0.25 and the identity takes 1 - x^2 for it, |x| < 0.25 here: at most 1/16 off, far less on average
        assert abs((losses[0] - losses[1]) / 2 - along) < 0.05 * np.sqrt((grads[i].double().cpu().numpy() ** 2 * step ** 2).sum()) + 0.03 * abs(along)


# ------------------------------------------------------------------------------------------ the cache


def _cache(torch, seed, lengths, page, kv_heads, dim, spare=2, spread=2.0):
    """A cache with shuffled pages, garbage (NaN too) wherever no key is; (tensors k, v, pages), (k, v per sequence as doubles)."""
    rng = np.random.default_rng(seed)
    most = max(1, -(-max(lengths) // page))
    count = len(lengths) * most + spare
    pages = rng.permutation(count)[:len(lengths) * most].reshape(len(lengths), most).astype(np.int32)
    k, v = (np.full((count, page, kv_heads, dim), np.nan) for _ in range(2))
    each = []
    for s, n in enumerate(lengths):
        ks, vs = _grid(rng, (n, kv_heads, dim), spread), rng.standard_normal((n, kv_heads, dim))
        for j in range(n):
            k[pages[s, j // page], j % page], v[pages[s, j // page], j % page] = ks[j], vs[j]
        each.append((ks, vs))
    k, v = _bf16(torch, k), _bf16(torch, v)
    each = [(ks, kcap_oracle.gather(v.float().cpu().numpy().astype(np.float64), pages[s], len(ks))) for s, (ks, _) in enumerate(each)]
    return (k, v, torch.from_numpy(pages).cuda()), each


LENGTHS = {"one token": [1], "ragged": [1, 2, 31, 32, 33, 127, 128, 129, 300], "some empty": [0, 40, 0, 700], "long": [2050, 5]}


@pytest.mark.parametrize("window", [0, 1, 50])
@pytest.mark.parametrize("page", [1, 16, 64])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (3, 3, 64), (40, 1, 64)])
def test_single_tokens_over_pages(gpu, lengths, page, heads, kv_heads, dim, window):
    binding, _, torch = gpu
    lengths = LENGTHS[lengths]
    (k, v, pages), each = _cache(torch, 10, lengths, page, kv_heads, dim)
    q64 = _grid(np.random.default_rng(11), (len(lengths), heads, dim), 2.0)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    options = dict(cap=32.0, scale=dim ** -0.5, window=window)
    o = binding.kcap_attention_paged(_bf16(torch, q64), k, v, pages, n, **options)
    for s, (ks, vs) in enumerate(each):
        want = kcap_oracle.attention(q64[s:s + 1], ks, vs, [0, 1], [0, len(ks)], **options)
        _near(o[s:s + 1], want["o"], want["o_off"], f"sequence {s}")


@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("cap,spread", [(32.0, 2.0), (64.0, 4.0), (64.0, 0.0)])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (40, 1, 64)])
def test_single_tokens_that_see_infinities(gpu, heads, kv_heads, dim, cap, spread, window):
    """A value that is infinite or NaN reaches its column of the rows that see it, as itself: weights are positive, whatever they are (all of them
    exactly 1 where spread is 0).  In texts of one share and of many, beside ones that a window hides; as pieces of one token too."""
    binding, _, torch = gpu
    lengths = [1, 40, 300, 3000, 129]
    (k, v, pages), each = _cache(torch, 48, lengths, 16, kv_heads, dim, spread=spread)
    rng = np.random.default_rng(49)
    for s, n in enumerate(lengths):
        for j in {n - 1, n // 2, max(n - 45, 0), 0}:
            for value in (np.inf, -np.inf, np.nan):
                head, columns = rng.integers(kv_heads), rng.integers(0, dim, 3)
                v[pages[s, j // 16].item(), j % 16, head, torch.from_numpy(columns).cuda()] = value
                each[s][1][j, head, columns] = value
    q64 = _grid(rng, (len(lengths), heads, dim), spread)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    options = dict(cap=cap, scale=dim ** -0.5, window=window)
    one = torch.arange(len(lengths) + 1, dtype=torch.int32, device="cuda")
    for what, o in (("single", binding.kcap_attention_paged(_bf16(torch, q64), k, v, pages, n, **options)),
                    ("pieces", binding.kcap_attention_paged(_bf16(torch, q64), k, v, pages, n, one, **options))):
        for s, (ks, vs) in enumerate(each):
            want = kcap_oracle.attention(q64[s:s + 1], ks, vs, [0, 1], [0, len(ks)], **options)
            assert np.isinf(want["o"]).any() and np.isnan(want["o"]).any()
            _near(o[s:s + 1], want["o"], want["o_off"], f"{what}, sequence {s}")


@pytest.mark.parametrize("window", [0, 45])
@pytest.mark.parametrize("page", [8, 128])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 2, 128), (3, 1, 64)])
def test_pieces_of_prompts_over_pages(gpu, page, heads, kv_heads, dim, window):
    binding, _, torch = gpu
    new, lengths = [1, 60, 0, 130, 7], [1, 200, 30, 130, 400]
    (k, v, pages), each = _cache(torch, 12, lengths, page, kv_heads, dim)
    at, at_np = _offsets(torch, new)
    q64 = _grid(np.random.default_rng(13), (sum(new), heads, dim), 2.0)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    options = dict(cap=32.0, scale=dim ** -0.5, window=window)
    o = binding.kcap_attention_paged(_bf16(torch, q64), k, v, pages, n, at, **options)
    for s, (ks, vs) in enumerate(each):
        rows = slice(at_np[s], at_np[s + 1])
        want = kcap_oracle.attention(q64[rows], ks, vs, [0, new[s]], [0, len(ks)], **options)
        _near(o[rows], want["o"], want["o_off"], f"sequence {s}")


def test_pieces_of_prompts_in_blocks_of_128_rows(gpu):
    test_pieces_of_prompts_over_pages(gpu, 16, 384, 2, 64, 0)
    test_pieces_of_prompts_over_pages(gpu, 8, 384, 3, 128, 33)


@pytest.mark.parametrize("heads", [4, 512])
def test_outputs_that_start_off_a_16_byte_line(gpu, heads):
    """Outputs need eight bytes only, with few heads and with many, and nothing next to them is written."""
    binding, _, torch = gpu
    (q, k, v), _ = _inputs(torch, 45, 133, 133, heads, 2, 64)
    at, _ = _offsets(torch, [100, 33])
    want_rest = torch.empty_like(q)
    want, _ = binding.kcap_attention(q, k, v, at, cap=50.0, rest=want_rest)
    rooms = [torch.full((q.numel() + 16,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out, rest = (room[4:4 + q.numel()].view(q.shape) for room in rooms)
    assert out.data_ptr() % 16 == 8
    binding.kcap_attention(q, k, v, at, cap=50.0, out=out, rest=rest)
    assert torch.equal(out, want) and torch.equal(rest, want_rest)
    assert all((room[:4] == 7).all() and (room[4 + q.numel():] == 7).all() for room in rooms)


@pytest.mark.parametrize("heads,kv_heads,dim,lengths", [(96, 4, 64, [1400, 600]), (96, 4, 128, [1400, 100]), (63, 7, 128, [2400, 131])])
def test_pieces_of_prompts_whose_keys_are_shared_out(gpu, heads, kv_heads, dim, lengths):
    """Few stretches of many rows behind long texts: blocks of 128 rows take parts of the keys, some of them empty in the shorter text."""
    binding, _, torch = gpu
    new = [130, 132]
    (k, v, pages), each = _cache(torch, 43, lengths, 16, kv_heads, dim)
    at, at_np = _offsets(torch, new)
    q64 = _grid(np.random.default_rng(44), (sum(new), heads, dim), 2.0)
    options = dict(cap=32.0, scale=dim ** -0.5)
    o = binding.kcap_attention_paged(_bf16(torch, q64), k, v, pages, torch.tensor(lengths, dtype=torch.int32, device="cuda"), at, **options)
    for s, (ks, vs) in enumerate(each):
        rows = slice(at_np[s], at_np[s + 1])
        want = kcap_oracle.attention(q64[rows], ks, vs, [0, new[s]], [0, len(ks)], **options)
        _near(o[rows], want["o"], want["o_off"], f"sequence {s}")


def test_wide_tables_and_layouts_of_the_cache(gpu):
    """64 intervals; heads before slots in a page, keys and values in one tensor, a table wider than its rows."""
    binding, _, torch = gpu
    lengths = [300, 77, 1000]
    (k, v, pages), each = _cache(torch, 14, lengths, 16, 2, 64)
    q64 = _grid(np.random.default_rng(15), (3, 6, 64), 2.0)
    q, n = _bf16(torch, q64), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    both = torch.stack([k, v], 1)                       # [pages, 2, page, heads, dim]
    heads_first = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v)]
    wider = torch.full((3, pages.shape[1] + 5), 1 << 20, dtype=torch.int32, device="cuda")
    wider[:, :pages.shape[1]] = pages
    options = dict(cap=50.0, scale=0.125)
    one = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    first = binding.kcap_attention64_paged(q, k, v, pages, n, **options)
    for s, (ks, vs) in enumerate(each):
        want = kcap_oracle.attention(q64[s:s + 1], ks, vs, [0, 1], [0, len(ks)], intervals=64, **options)
        _near(first[s:s + 1], want["o"], want["o_off"], f"sequence {s}")
        many = binding.kcap_attention64_paged(q, k, v, pages, n, one, **options)
        _near(many[s:s + 1], want["o"], want["o_off"], f"sequence {s}, as a piece of a prompt")
    for kc, vc, table in ((both[:, 0], both[:, 1], pages), (*heads_first, pages), (k, v, wider), (k, v, wider[:, :pages.shape[1]])):
        got = binding.kcap_attention64_paged(q, kc, vc, table, n, **options)
        assert torch.allclose(got.float(), first.float(), rtol=2 ** -7, atol=1e-3)


def test_a_long_cache_past_32_bits(gpu):
    """Pages behind 2^32 bytes and 2^31 elements of the cache."""
    binding, _, torch = gpu
    page, kv_heads, dim = 64, 8, 128
    count = (1 << 31) // (page * kv_heads * dim) + 300
    k, v = (torch.zeros((count, page, kv_heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rng = np.random.default_rng(16)
    pages = torch.tensor([[count - 1, 3, count - 5]], dtype=torch.int32, device="cuda")
    cos = torch.ones((192, 64), device="cuda")
    new_k, new_v = (_bf16(torch, _grid(rng, (150, kv_heads, dim), 2.0)) for _ in range(2))
    q = _bf16(torch, _grid(rng, (150, 8, dim), 2.0))
    at = torch.tensor([0, 150], dtype=torch.int32, device="cuda")
    binding.kcap_append(q, new_k, new_v, k, v, pages, torch.zeros(1, dtype=torch.int32, device="cuda"), at, cos=cos, sin=torch.zeros_like(cos))
    assert torch.equal(k[count - 1], new_k[:64]) and torch.equal(k[3], new_k[64:128]) and torch.equal(v[count - 5, :22], new_v[128:])
    n = torch.tensor([150], dtype=torch.int32, device="cuda")
    one = binding.kcap_attention_paged(q[-1:], k, v, pages, n, cap=50.0)
    all_ = binding.kcap_attention_paged(q, k, v, pages, n, at, cap=50.0)
    flat, _ = binding.kcap_attention(q, new_k, new_v, at, cap=50.0)
    assert torch.equal(all_, flat)
    q64, k64, v64 = (t.double().cpu().numpy() for t in (q[-1:], new_k, new_v))
    want = kcap_oracle.attention(q64, k64, v64, [0, 1], [0, 150], cap=50.0, scale=dim ** -0.5)
    _near(one, want["o"], want["o_off"], "one token")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("angles", [8, 32, 64])
@pytest.mark.parametrize("page", [1, 16])
def test_append(gpu, interleaved, angles, page):
    """Keys and queries turned, values and the rest as they are, in their places and nowhere else; parts of heads turned."""
    binding, _, torch = gpu
    dim, heads, kv_heads = 128, 6, 2
    rng = np.random.default_rng(17)
    before, new = [0, 13, 40, 7], [20, 1, 0, 30]
    most = -(-60 // page)
    count = 4 * most + 3
    pages = rng.permutation(count)[:4 * most].reshape(4, most).astype(np.int32)
    q, k, v = (_bf16(torch, rng.standard_normal((sum(new), h, dim))) for h in (heads, kv_heads, kv_heads))
    caches = [torch.full((count, page, kv_heads, dim), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    angle = np.outer(np.arange(64), 10000.0 ** (-np.arange(angles) / angles))
    cos, sin = (torch.from_numpy(f(angle).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    at, at_np = _offsets(torch, new)
    n = torch.tensor(before, dtype=torch.int32, device="cuda")
    out = binding.kcap_append(q, k, v, *caches, torch.from_numpy(pages).cuda(), n, at, cos=cos, sin=sin, interleaved=interleaved)
    wide = [t.float().cpu().numpy().astype(np.float64) for t in (q, k, v)]
    want_q = np.zeros(wide[0].shape)
    want = [np.full(c.shape, 9.0) for c in caches]
    c64, s64 = cos.double().cpu().numpy(), sin.double().cpu().numpy()
    for s in range(4):
        for i in range(new[s]):
            row, place = at_np[s] + i, before[s] + i
            want_q[row] = kcap_oracle.turned(wide[0][row], c64[place], s64[place], interleaved)
            spot = pages[s, place // page], place % page
            want[0][spot] = kcap_oracle.turned(wide[1][row], c64[place], s64[place], interleaved)
            want[1][spot] = wide[2][row]
    # two products, a sum and the rounding of the result
    for got, exact, size in ((out, want_q, np.abs(wide[0]).max()), (caches[0], want[0], np.abs(wide[1]).max()), (caches[1], want[1], 0.0)):
        _near(got, exact, kcap_oracle.HALF * np.abs(exact) + 4 * 2.0 ** -24 * size + 1e-30, "append")


def test_append_in_place_one_token_each_and_tokens_without_a_place(gpu):
    binding, _, torch = gpu
    rng = np.random.default_rng(18)
    q, k, v = (_bf16(torch, rng.standard_normal((5, h, 64))) for h in (4, 2, 2))
    pages = torch.tensor([[0, 1], [2, 3], [4, 99], [5, -1], [6, 7]], dtype=torch.int32, device="cuda")
    #      in page 0 | past the table | page 99 is none | page -1 is none | no angles
    before = torch.tensor([3, 32, 16, 20, 25], dtype=torch.int32, device="cuda")
    angle = np.outer(np.arange(25), 0.1 * np.arange(32))
    cos, sin = (torch.from_numpy(f(angle).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    caches = [torch.full((8, 16, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    turned = q.clone()
    assert binding.kcap_append(turned, k, v, *caches, pages, before, cos=cos, sin=sin, out=turned) is turned
    assert torch.equal(binding.kcap_append(q, k, v, *caches, pages, before, cos=cos, sin=sin).view(torch.int16), turned.view(torch.int16))
    assert torch.equal(caches[1][0, 3], v[0])
    caches[0][0, 3], caches[1][0, 3] = 9.0, 9.0
    assert all((c == 9).all() for c in caches)
    assert turned[[1, 4]].isnan().all() and not turned[[0, 2, 3]].isnan().any()


# ------------------------------------------------------------------------------------- the host path


def _both_paths(binding, call):
    """What a call gives through the C++ host path and through the Python code."""
    assert binding._host is not None
    patch = pytest.MonkeyPatch()
    taken = call()
    patch.setattr(binding, "_host", None)
    patch.setattr(binding, "_calls", {})
    try:
        return taken, call()
    finally:
        patch.undo()


def test_host_path_and_python_code_give_the_same(gpu):
    binding, autograd, torch = gpu
    (q, k, v), _ = _inputs(torch, 31, 90, 90, 4, 2, 64)
    do = _bf16(torch, np.random.default_rng(32).standard_normal((90, 4, 64)))
    at, _ = _offsets(torch, [30, 60])
    (kc, vc, pages), _ = _cache(torch, 33, [300, 40], 16, 2, 64)
    n = torch.tensor([300, 40], dtype=torch.int32, device="cuda")
    two = torch.tensor([0, 5, 6], dtype=torch.int32, device="cuda")
    cos, sin = torch.rand((400, 32), device="cuda"), torch.rand((400, 32), device="cuda")
    fused = torch.cat([q, k, v], 1)
    rest = torch.empty_like(q)

    def train(**options):
        leaves = [t.detach().clone().requires_grad_() for t in (q, k, v)]
        o = autograd.kcap_attention(*leaves, at, **options)
        return (o, *torch.autograd.grad(o, leaves, do))
    lut32, lut64 = binding.ktanh_fit_lut_bmin0(), binding.ktanh_fit_lut64()
    calls = [
        lambda: binding.kcap_attention(q, k, v, at, cap=50.0),
        lambda: binding.kcap_attention(q, k, v, at, at, cap=30, scale=0.25, causal=False, window=9, lut=lut32),
        lambda: (*binding.kcap_attention64(q, k, v, at, cap=50.0, lut=lut64, out=torch.empty_like(q), rest=rest), rest.clone()),
        lambda: binding.kcap_attention(fused[:, :4], fused[:, 4:6], fused[:, 6:], at, cap=50.0),
        lambda: (binding.kcap_attention_paged(q[:2], kc, vc, pages, n, cap=50.0),),
        lambda: (binding.kcap_attention64_paged(q[:6], kc, vc, pages, n, two, cap=50.0, scale=0.1, window=33),),
        lambda: (binding.kcap_append(q[:2], k[:2], v[:2], kc, vc, pages, n - 1, cos=cos, sin=sin), kc.clone(), vc.clone()),
        lambda: (binding.kcap_append(q[:6], k[:6], v[:6], kc, vc, pages, n - 9, two, cos=cos, sin=sin, interleaved=True), kc.clone(), vc.clone()),
        lambda: train(cap=50.0), lambda: train(cap=30.0, scale=0.3, causal=False, window=20, intervals=64),
    ]
    for i, call in enumerate(calls):
        fast, slow = _both_paths(binding, call)
        assert len(fast) == len(slow)
        for a, b in zip(fast, slow):
            assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride() and a.requires_grad == b.requires_grad, i
            assert torch.equal(a.detach().view(torch.int16), b.detach().view(torch.int16)), i
    host = binding._host
    assert host.cap_attention(q, k, v, at, at, 50.0, None, True, 0, None, None, None, None, False) is not None
    assert host.cap_attention_paged(q[:2], kc, vc, pages, n, None, 50.0, None, 0, None, None, True) is not None
    assert host.cap_append(q[:2], k[:2], v[:2], kc, vc, pages, n - 1, None, cos, sin, False, None) is not None
    leaf = q.clone().requires_grad_()
    assert host.train_cap_attention(leaf, k, v, at, at, 50.0, None, True, 0, False) is not None
    # and what is not ordinary is left to the Python code
    assert host.cap_attention(q.float(), k, v, at, at, 50.0, None, True, 0, None, None, None, None, False) is None
    assert host.cap_attention(q, k, v, at, at, "50", None, True, 0, None, None, None, None, False) is None
    assert host.cap_attention(q, k, v, at, at[:1], 50.0, None, True, 0, None, None, None, None, False) is None
    assert host.cap_attention(q[:, :3], k, v, at, at, 50.0, None, True, 0, None, None, None, None, False) is None
    assert host.train_cap_attention(q, k, v, at, at, 50.0, None, True, 0, False) is None
    with pytest.raises(binding.KtanhError) as err:
        binding.kcap_attention(q, k, v, at, cap=80.0)
    assert err.value.status == 4


# ----------------------------------------------------------------------------------------- refusals


def test_refusals(gpu):
    binding, _, torch = gpu
    q, k, v = (torch.zeros((8, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    at = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        binding.kcap_attention(q.float(), k, v, at, cap=50.0)
    with pytest.raises(TypeError):
        binding.kcap_attention(q, k, v, at.long(), cap=50.0)
    with pytest.raises(ValueError):
        binding.kcap_attention(q.cpu(), k, v, at, cap=50.0)
    with pytest.raises(ValueError):
        binding.kcap_attention(q, k[:, :, ::2], v[:, :, ::2], at, cap=50.0)
    with pytest.raises(ValueError):
        binding.kcap_attention(q[:, :3], k, v, at, cap=50.0)
    with pytest.raises(ValueError):
        binding.kcap_attention(q, k, v[:4], at, cap=50.0)
    with pytest.raises(ValueError):
        binding.kcap_attention(q, k, v, at, cap=50.0, window=-1)
    with pytest.raises(ValueError):
        binding.kcap_attention(q, k, v, at, cap=50.0, out=torch.empty_like(q)[:4])
    for bad in (0.0, -1.0, 65.0, float("nan"), float("inf")):
        with pytest.raises(binding.KtanhError) as err:
            binding.kcap_attention(q, k, v, at, cap=bad)
        assert err.value.status == 4
    with pytest.raises(binding.KtanhError) as err:
        binding.kcap_attention(q, k, v, at, cap=50.0, scale=float("inf"))
    assert err.value.status == 4
    narrow = [t[..., :32] for t in (q, k, v)]
    with pytest.raises(binding.KtanhError) as err:
        binding.kcap_attention(*narrow, at, cap=50.0)
    assert err.value.status == 4
    off = torch.zeros(8 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(8, 4, 64)
    with pytest.raises(binding.KtanhError) as err:
        binding.kcap_attention(off, k, v, at, cap=50.0)
    assert err.value.status == 2
    rows = binding.ktanh_default_lut().as_tuples()
    rows[31] = (127, 4, 110)                            # a valid table, but K up to 1.9
    with pytest.raises(binding.KtanhError) as err:
        binding.kcap_attention(q, k, v, at, cap=50.0, lut=binding.KtanhLut.from_tuples(rows))
    assert err.value.status == 3
    caches = [torch.zeros((4, 12, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pages, n = torch.zeros((8, 2), dtype=torch.int32, device="cuda"), torch.ones(8, dtype=torch.int32, device="cuda")
    with pytest.raises(binding.KtanhError) as err:      # twelve slots in a page
        binding.kcap_attention_paged(q, *caches, pages, n, cap=50.0)
    assert err.value.status == 4
    good = [c[:, :8] for c in caches]
    with pytest.raises(ValueError):
        binding.kcap_attention_paged(q, *good, pages[:4], n, cap=50.0)
    with pytest.raises(ValueError):
        binding.kcap_attention_paged(q, *good, pages, n[:4], cap=50.0)
    with pytest.raises(TypeError):
        binding.kcap_attention_paged(q, *good, pages.long(), n, cap=50.0)
    cos = torch.ones((16, 12), device="cuda")
    with pytest.raises(binding.KtanhError) as err:      # twelve angles
        binding.kcap_append(q, k, v, *good, pages, n, cos=cos, sin=cos)
    assert err.value.status == 4
    with pytest.raises(ValueError):
        binding.kcap_append(q, k, v, *good, pages, n, cos=cos, sin=cos[:3])
    empty = binding.kcap_attention(q[:0], k[:0], v[:0], torch.zeros(1, dtype=torch.int32, device="cuda"), cap=50.0)
    assert empty[0].shape == (0, 4, 64) and empty[1].shape == (4, 0)


# ------------------------------------------------------------------------------------- no documents


def test_rows_without_any_document(gpu):
    """Offsets of no document at all beside tensors that have rows: all of them are rows of no document, and their results are zero."""
    binding, autograd, torch = gpu
    (q, k, v), _ = _inputs(torch, 50, 70, 90, 4, 2, 64)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()

    def held(shape, dtype=torch.bfloat16):
        return torch.full(shape, 7.0, dtype=dtype, device="cuda")
    for attend, backward in ((binding.kcap_attention, binding.kcap_attention_backward), (binding.kcap_attention64, binding.kcap_attention64_backward)):
        for stream in (None, side):
            side.wait_stream(torch.cuda.current_stream())
            out, lse, rest = held(q.shape), held((4, 70), torch.float32), held(q.shape)
            side.wait_stream(torch.cuda.current_stream())
            o, sums = attend(q, k, v, none, cap=50.0, out=out, lse=lse, rest=rest, stream=stream)
            torch.cuda.synchronize()
            assert o is out and sums is lse and not o.any() and not rest.any() and (lse == -float("inf")).all()
            grads = [held(t.shape) for t in (q, k, v)]
            side.wait_stream(torch.cuda.current_stream())
            got = backward(held(q.shape), q, k, v, o, lse, none, cap=50.0, dq=grads[0], dk=grads[1], dv=grads[2], rest=rest, stream=stream)
            torch.cuda.synchronize()
            assert all(a is b and not a.any() for a, b in zip(got, grads))
    for intervals in (32, 64):
        leaves = [t.clone().requires_grad_() for t in (q, k, v)]
        o = autograd.kcap_attention(*leaves, none, cap=50.0, intervals=intervals)
        assert not o.any() and not any(t.any() for t in torch.autograd.grad(o, leaves, torch.ones_like(o)))
    cache = torch.ones((4, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    pages, lengths = torch.zeros((0, 3), dtype=torch.int32, device="cuda"), none[:0]
    for paged in (binding.kcap_attention_paged, binding.kcap_attention64_paged):
        for stream in (None, side):
            out = held(q.shape)
            side.wait_stream(torch.cuda.current_stream())
            assert paged(q, cache, cache, pages, lengths, none, cap=50.0, out=out, stream=stream) is out
            torch.cuda.synchronize()
            assert not out.any()
        assert not paged(q, cache, cache, pages, lengths, none, cap=50.0).any()
    assert paged(q[:0], cache, cache, pages, lengths, cap=50.0).shape == (0, 4, 64)
    cos = torch.ones((16, 32), device="cuda")
    turned = held(q.shape)          # rows of no sequence are left as they are
    binding.kcap_append(q, k[:70], v[:70], cache, cache, pages, lengths, none, cos=cos, sin=cos, out=turned)
    assert (turned == 7).all() and (cache == 1).all()
