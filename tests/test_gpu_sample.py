"""The choice of the next token against its definition in 64 bits, row by row in numpy: equal tokens."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1909_07729_amd import binding
    torch.cuda.set_device(0)
    return torch, binding


def _ranked(z, temperature, top_k, top_p, min_p):
    """(tokens by rank, G of the kept ones): the definition on one row of Float32 logits."""
    order = np.argsort(-z, kind="stable")
    n = len(z)
    if temperature <= 0:
        return order, np.ones(1)
    with np.errstate(all="ignore"):
        a = np.where(z[order] == z[order[0]], 0.0, (z[order[0]].astype(np.float64) - z[order]) / np.float64(np.float32(temperature)))
        w = np.where(np.isnan(a), 0.0, np.exp(-a))
    mass = np.cumsum(w)
    kept = n if top_k <= 0 or top_k > n else top_k
    limit = np.float64(np.float32(top_p)) * mass[kept - 1]
    kept = min(kept, int((np.concatenate([[0], mass[:-1]]) < limit).sum()))
    kept = min(kept, int((w >= np.float64(np.float32(min_p))).sum()))
    return order, mass[:max(kept, 1)]


def _token(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    if np.isnan(z).any() or (z == -np.inf).all():
        return -1
    order, mass = _ranked(z, temperature, top_k, top_p, min_p)
    return int(order[min(int((mass <= np.float64(u) * mass[-1]).sum()), len(mass) - 1)])


def _capped(oracle, z, cap, wide):
    """cap * Kf(z / cap) in Float32; masked tokens stay masked."""
    x = (z / np.float32(cap)).astype(np.float32)
    k = getattr(oracle, "ktanh64_f32" if wide else "ktanh_f32")(x.reshape(-1).view(np.uint32)).view(np.float32).reshape(x.shape)
    return np.where(z == -np.inf, z, np.float32(cap) * k).astype(np.float32)


def _logits(torch, rows, vocabulary, dtype, seed, spread=3.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (torch.randn((rows, vocabulary), generator=gen, device="cuda") * spread).to(getattr(torch, dtype))


def _uniform(torch, rows, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1000)
    return torch.rand(rows, generator=gen, device="cuda")


SETTINGS = [dict(), dict(temperature=0.0), dict(top_k=1), dict(top_k=5), dict(top_k=50, top_p=0.95), dict(top_p=0.9), dict(top_p=0.0), dict(min_p=0.05),
            dict(temperature=1.5, top_k=3000), dict(temperature=0.7, top_p=0.99, min_p=0.001), dict(temperature=20.0), dict(temperature=20.0, top_p=0.7, top_k=9000),
            dict(temperature=0.05), dict(min_p=1.0), dict(temperature=30.0, top_p=0.3, min_p=0.9)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocabulary", [1, 2, 7, 64, 1000, 2048, 2049, 5000, 32000, 50257, 131072])
def test_settings(gpu, dtype, vocabulary):
    torch, binding = gpu
    rows = 6
    for i, settings in enumerate(SETTINGS):
        logits, u = _logits(torch, rows, vocabulary, dtype, 100 * vocabulary + i), _uniform(torch, rows, i)
        got = binding.ksample(logits, u, **settings)
        z, un = logits.float().cpu().numpy(), u.cpu().numpy()
        assert got.tolist() == [_token(z[r], un[r], **settings) for r in range(rows)], settings


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows, vocabulary", [(64, 300), (17, 40000), (3, 200000)])
def test_settings_of_each_row(gpu, dtype, rows, vocabulary):
    torch, binding = gpu
    rng = np.random.default_rng(rows)
    logits, u = _logits(torch, rows, vocabulary, dtype, rows), _uniform(torch, rows, 1)
    values = {"temperature": rng.choice([0.0, 0.5, 1.0, 8.0, -1.0], rows).astype(np.float32), "top_k": rng.choice([0, 1, 10, 2500, -3, 10 ** 9], rows).astype(np.int32),
              "top_p": rng.choice([1.0, 0.9, 0.5, 0.0], rows).astype(np.float32), "min_p": rng.choice([0.0, 0.01, 0.3], rows).astype(np.float32)}
    got = binding.ksample(logits, u, **{n: torch.from_numpy(v).cuda() for n, v in values.items()})
    z, un = logits.float().cpu().numpy(), u.cpu().numpy()
    assert got.tolist() == [_token(z[r], un[r], **{n: v[r].item() for n, v in values.items()}) for r in range(rows)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows, vocabulary", [(61, 40001), (60, 65536), (33, 70003), (259, 33000)])
def test_many_long_rows(gpu, dtype, rows, vocabulary):
    """Chunks of 32768 logits, the last of a row full, short or of one vector; greedy rows, empty ones and others in one call, twice with the same workspace."""
    torch, binding = gpu
    rng = np.random.default_rng(vocabulary)
    logits, u = _logits(torch, rows, vocabulary, dtype, rows), _uniform(torch, rows, 1)
    logits[3] = -float("inf")
    logits[4, -1] = float("nan")
    logits[5, :-1] = -float("inf")
    logits[6, : vocabulary // 2] = -float("inf")
    values = {"temperature": rng.choice([0.0, 0.5, 1.0, 8.0], rows).astype(np.float32), "top_k": rng.choice([0, 0, 1, 40, 5000], rows).astype(np.int32),
              "top_p": rng.choice([1.0, 0.9, 0.5], rows).astype(np.float32), "min_p": rng.choice([0.0, 0.0, 0.02], rows).astype(np.float32)}
    settings = {n: torch.from_numpy(v).cuda() for n, v in values.items()}
    z, un = logits.float().cpu().numpy(), u.cpu().numpy()
    want = [_token(z[r], un[r], **{n: v[r].item() for n, v in values.items()}) for r in range(rows)]
    assert want[3] == want[4] == -1 and want[5] == vocabulary - 1
    graph, out = torch.cuda.CUDAGraph(), torch.empty(rows, dtype=torch.int64, device="cuda")
    binding.ksample(logits, u, out=out, **settings)
    assert out.tolist() == want
    with torch.cuda.graph(graph):
        binding.ksample(logits, u, out=out, **settings)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert out.tolist() == want


@pytest.mark.parametrize("vocabulary", [100, 1500, 9000, 32768])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_few_tokens_of_top_k(gpu, oracle, vocabulary, cap):
    """What top-k leaves with others near it: ties over its end, masked tokens, rows with fewer tokens than it asks for, every other setting behind it."""
    torch, binding = gpu
    logits = _logits(torch, 7, vocabulary, "float32", vocabulary)
    logits[1] = logits[1].round()
    logits[2, torch.arange(vocabulary, device="cuda") % 3 != 0] = -float("inf")
    logits[3, 10:] = -float("inf")
    logits[4] = logits[4] * 1e-4 + 5
    logits[5] = 0
    logits[5, : vocabulary // 4] = -700.0               # of no weight
    z = logits.cpu().numpy() if cap == 0 else _capped(oracle, logits.cpu().numpy(), cap, False)
    for i, settings in enumerate([dict(top_k=2), dict(top_k=30), dict(top_k=60, top_p=0.8), dict(top_k=40, min_p=0.3), dict(top_k=500, temperature=4.0, top_p=0.97, min_p=0.01),
                                  dict(top_k=513), dict(top_k=99, temperature=0.02), dict(top_k=20, top_p=0.0), dict(top_k=45, min_p=1.0)]):
        u = _uniform(torch, 7, i)
        un = u.cpu().numpy()
        got = binding.ksample(logits, u, cap=cap, **settings).tolist()
        assert got == [_token(z[r], un[r], **settings) for r in range(7)], settings


@pytest.mark.parametrize("vocabulary", [3000, 30000, 70000])
def test_ties_flat_rows_and_outliers(gpu, vocabulary):
    """Rows that crowd one bin: equal logits, two values, a flat row under one outlier, differences at the last bit."""
    torch, binding = gpu
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    flat = torch.zeros(vocabulary, device="cuda")
    two = (torch.rand(vocabulary, generator=gen, device="cuda") < 0.5).float()
    outlier = flat.clone()
    outlier[vocabulary // 3] = 25.0
    close = 1.0 + torch.randint(0, 40, (vocabulary,), generator=gen, device="cuda") * 2.0 ** -23
    low = torch.randn(vocabulary, generator=gen, device="cuda") * 1e-3
    low[5] = -30.0
    signed = torch.where(torch.rand(vocabulary, generator=gen, device="cuda") < 0.5, 0.0, -0.0)
    logits = torch.stack([flat, two, outlier, close, low, signed])
    z = logits.cpu().numpy()
    for seed, settings in enumerate([dict(), dict(top_k=7), dict(top_k=2600), dict(top_p=0.5), dict(top_k=2700, top_p=0.9), dict(min_p=0.5), dict(temperature=25.0, top_p=0.6)]):
        for u in (0.0, 0.25, 0.9999999):
            got = binding.ksample(logits, torch.full((6,), u, device="cuda"), **settings)
            assert got.tolist() == [_token(z[r], np.float32(u), **settings) for r in range(6)], (settings, u)


def test_masks_infinities_and_nans(gpu):
    torch, binding = gpu
    vocabulary, inf, nan = 4000, float("inf"), float("nan")
    logits = _logits(torch, 12, vocabulary, "float32", 1)
    logits[0] = -inf                                    # nothing to choose from
    logits[1, 17] = nan
    logits[2, :] = -inf
    logits[2, 3999] = -50.0                             # one token
    logits[3, ::2] = -inf
    logits[4, 100] = inf
    logits[5, 7], logits[5, 3000] = inf, inf
    logits[6] = torch.finfo(torch.float32).min          # the type's lowest value is a value
    logits[7, 1:] = torch.finfo(torch.float32).min
    logits[8, :2000] = torch.finfo(torch.float32).min
    logits[9, 5] = 3e38
    logits[10, -1] = -nan
    u = _uniform(torch, 12, 2)
    z, un = logits.cpu().numpy(), u.cpu().numpy()
    for settings in (dict(), dict(top_k=20, top_p=0.9), dict(temperature=0.0), dict(min_p=0.1), dict(top_p=0.95)):
        got = binding.ksample(logits, u, **settings).tolist()
        assert got == [_token(z[r], un[r], **settings) for r in range(12)], settings
        assert got[0] == got[1] == got[10] == -1 and got[2] == 3999 and got[3] % 2 and got[4] == 100 and got[5] in (7, 3000)
    half = logits.bfloat16()                            # the lowest value rounds to -infinity there
    z = half.float().cpu().numpy()
    assert binding.ksample(half, u, top_p=0.9).tolist() == [_token(z[r], un[r], top_p=0.9) for r in range(12)]


def test_uniform_numbers_at_the_ends_and_beyond(gpu):
    torch, binding = gpu
    logits = _logits(torch, 1, 5000, "float32", 4).expand(7, -1)        # rows with a stride of 0
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -1.0, float("nan"), 2.0 ** -149], device="cuda")
    z = logits[0].cpu().numpy()
    for settings in (dict(top_k=10), dict(), dict(top_p=0.5)):
        got = binding.ksample(logits, u, **settings).tolist()
        first, last = _token(z, 0.0, **settings), _token(z, 1.0, **settings)
        assert got[0] == got[4] == got[5] == first and got[6] == _token(z, 2.0 ** -149, **settings)
        assert got[2] == got[3] == last
        assert got[1] == _token(z, 1.0 - 2.0 ** -24, **settings)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_capped_logits(gpu, oracle, dtype, wide):
    torch, binding = gpu
    for vocabulary, cap in ((700, 30.0), (33000, 30.0), (33000, 5.0)):
        logits, u = _logits(torch, 8, vocabulary, dtype, vocabulary, 6.0), _uniform(torch, 8, 5)
        logits[1, ::3] = -float("inf")
        logits[2, 9] = float("inf")                     # capped like any other
        logits[3, 9] = float("nan")
        z = _capped(oracle, logits.float().cpu().numpy(), cap, wide)
        for settings in (dict(), dict(top_k=40, top_p=0.9), dict(temperature=0.0), dict(top_p=0.8, temperature=0.6), dict(min_p=0.3)):
            got = (binding.ksample64 if wide else binding.ksample)(logits, u, cap=cap, **settings)
            assert got.tolist() == [_token(z[r], u[r].item(), **settings) for r in range(8)], (vocabulary, cap, settings)
    table = binding.ktanh_fit_lut64() if wide else binding.ktanh_fit_lut()
    again = (binding.ksample64 if wide else binding.ksample)(logits, u, cap=cap, min_p=0.3, lut=table)
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_alignment(gpu, dtype):
    torch, binding = gpu
    wide = _logits(torch, 9, 3333, dtype, 6)
    u = _uniform(torch, 9, 6)
    for part in (wide[:, 1:], wide[:, 8:3008], wide[::2, 3:2900], wide.flatten()[5:5 + 8 * 3333].view(8, 3333)):
        assert torch.equal(binding.ksample(part, u[:len(part)], top_p=0.9), binding.ksample(part.contiguous(), u[:len(part)], top_p=0.9))


def test_frequencies(gpu):
    """70000 draws over 5 tokens.  A frequency f has a standard deviation of at most 0.5 / sqrt(70000) = 0.0019; five of them are allowed."""
    torch, binding = gpu
    logits = torch.tensor([0.5, 2.0, -1.0, 1.0, 0.0], device="cuda").expand(70000, -1)
    tokens = binding.ksample(logits, _uniform(torch, 70000, 7), temperature=0.8)
    want = torch.softmax(logits[0].double() / 0.8, 0)
    assert (torch.bincount(tokens, minlength=5) / 70000 - want).abs().max() < 5 * 0.0019


def test_graphs_streams_and_outputs(gpu):
    torch, binding = gpu
    logits, u = _logits(torch, 5, 9000, "bfloat16", 8), _uniform(torch, 5, 8)
    out = torch.full((5,), 77, dtype=torch.int64, device="cuda")
    assert binding.ksample(logits, u, out=out) is out
    kinds = [dict(top_k=40), dict(top_p=0.9), dict()]
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            made = [binding.ksample(logits, u, **k) for k in kinds]
        graphs.append((graph, made))
    for seed in range(3):
        logits.copy_(_logits(torch, 5, 9000, "bfloat16", 20 + seed))
        u.copy_(_uniform(torch, 5, 30 + seed))
        want = [binding.ksample(logits, u, **k) for k in kinds]
        for graph, made in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(made, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    one = binding.ksample(logits, u, **kinds[1], stream=side)
    side.synchronize()
    assert torch.equal(one, want[1])
    assert binding.ksample(logits[:0], u[:0]).shape == (0,)


def test_both_host_paths_give_the_same_and_refuse(gpu, monkeypatch):
    """Ordinary calls go through C++ where it is built, others through Python."""
    torch, binding = gpu
    assert binding._host is not None
    logits, u = _logits(torch, 6, 5000, "bfloat16", 9)[:, 3:], _uniform(torch, 6, 9)
    each = {"temperature": torch.full((6,), 0.7, device="cuda"), "top_k": torch.full((6,), 30, dtype=torch.int32, device="cuda"),
            "top_p": torch.full((6,), 0.9, device="cuda"), "min_p": torch.full((6,), 0.01, device="cuda")}
    results = []
    for host in (binding._host, None):
        monkeypatch.setattr(binding, "_host", host)
        results.append([binding.ksample(logits, u), binding.ksample(logits.float(), u, temperature=0.7, top_k=30, top_p=0.9, min_p=0.01),
                        binding.ksample(logits, u, **each), binding.ksample64(logits, u, cap=30, top_p=1), binding.ksample(logits, u, top_k=10 ** 12)])
        for bad, error in ((dict(temperature=-1.0), binding.KtanhError), (dict(top_p=1.5), binding.KtanhError), (dict(cap=-3.0), binding.KtanhError),
                           (dict(top_k=-1), ValueError), (dict(top_k=2.5), TypeError), (dict(temperature=each["temperature"][:3]), ValueError),
                           (dict(top_k=each["top_p"]), TypeError), (dict(out=torch.empty(6, device="cuda")), TypeError)):
            with pytest.raises(error):
                binding.ksample(logits, u, **bad)
        monkeypatch.undo()
    assert all(torch.equal(a, b) for a, b in zip(*results)) and torch.equal(results[0][1], results[0][2])
    with pytest.raises(ValueError):
        binding.ksample(logits, u[:5])
    with pytest.raises(binding.KtanhError):
        binding.ksample(logits[:, :0], u)
