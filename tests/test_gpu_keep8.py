"""Swish and GELU that keep their input in 8 bits, against the oracle's activations and gradients at the values that the codes stand for:
identical bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

NAMES = [f"k{a}{w}{t}" for a in ("swish", "gelu") for w in ("", "64") for t in ("", "_f32")]


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1909_07729_amd import binding
    torch.cuda.set_device(0)
    return torch, binding


def _bf16(x):
    """Float32 to BFloat16 patterns, to nearest even; NaN stays one."""
    u = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    out = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), out)


def _wide(p):
    return (p.astype(np.uint32) << 16).view(np.float32)


def _checkpoint(x):
    """(codes, scales) of Float32 values, by the definition."""
    n = len(x)
    rows = np.pad(x, (0, -n % 128)).reshape(-1, 128)
    finite = np.isfinite(rows)
    top = np.where(finite, np.abs(rows), 0).max(1, keepdims=True).astype(np.float32)
    tiny = top < np.float32(2.0 ** -120)
    with np.errstate(all="ignore"):
        inverse = np.where(tiny, np.float32(0), np.float32(127) / top).astype(np.float32)
        codes = np.where(finite, np.rint(rows * inverse), -128).astype(np.int8)
    scales = np.where(tiny, np.float32(0), top / np.float32(127)).astype(np.float32)
    return codes.reshape(-1)[:n], scales[:, 0]


def _restored(codes, scales, f32):
    """What the codes stand for, as patterns of the tensor's type."""
    x = codes.astype(np.float32) * np.repeat(scales, 128)[:len(codes)]
    x = np.where(codes == -128, np.float32(np.nan), x).astype(np.float32)
    return x.view(np.uint32) if f32 else _bf16(x)


def _same(got, want, f32):
    """Identical bits, NaNs as a class."""
    mask, inf = (0x7FFFFFFF, 0x7F800000) if f32 else (0x7FFF, 0x7F80)
    nan = (want & mask) > inf
    assert np.array_equal((got & mask) > inf, nan)
    assert np.array_equal(got[~nan], want[~nan])


def _arrays(torch, t, f32):
    return t.detach().flatten().view(torch.int32 if f32 else torch.int16).cpu().numpy().view(np.uint32 if f32 else np.uint16)


def _tensor(torch, patterns, f32, offset=0):
    """On the GPU, `offset` elements into its memory."""
    kind, view = (np.int32, torch.float32) if f32 else (np.int16, torch.bfloat16)
    room = torch.empty(len(patterns) + offset, dtype=view, device="cuda")
    room[offset:].view(torch.int32 if f32 else torch.int16).copy_(torch.from_numpy(patterns.view(kind).copy()))
    return room[offset:]


def _values(n, f32, seed, special):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal(n) * np.exp(rng.uniform(-3, 2, (n + 99) // 100).repeat(100)[:n])).astype(np.float32)
    if special and n > 600:
        x[3], x[200], x[201] = np.nan, np.inf, -np.inf
        x[256:384] = 0.0
        x[384:512] = np.float32(2.0 ** -121)            # below the smallest group that has a scale
        x[512:600] = np.float32(1e-40)
        if n > 1500:
            x[640:768] *= np.float32(2.0 ** -118)
            x[768:896] = np.float32(3e38) * np.sign(x[768:896])
            x[896:1024] = np.inf                        # no finite value in the group
            x[1024:1152:2] = -0.0
    dy = rng.standard_normal(n).astype(np.float32)
    return (x.view(np.uint32), dy.view(np.uint32)) if f32 else (_bf16(x), _bf16(dy))


def _oracle(oracle, name, f32, *args):
    out = getattr(oracle, name)(*((a.view(np.float32) for a in args) if f32 else args))
    return out.view(np.uint32) if f32 else out


def _check(gpu, oracle, name, n, seed, special=False, offset=0, code_offset=0):
    torch, binding = gpu
    f32 = name.endswith("_f32")
    xp, dyp = _values(n, f32, seed, special)
    x, dy = _tensor(torch, xp, f32, offset), _tensor(torch, dyp, f32, offset)
    out = _tensor(torch, np.zeros_like(xp), f32, offset)
    codes = torch.zeros(n + code_offset, dtype=torch.int8, device="cuda")[code_offset:]
    y, codes, scales = getattr(binding, name + "_keep8")(x, out=out, codes=codes)
    want_codes, want_scales = _checkpoint(xp.view(np.float32) if f32 else _wide(xp))
    assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)
    _same(_arrays(torch, y, f32), _oracle(oracle, name, f32, xp), f32)
    x8 = _restored(want_codes, want_scales, f32)
    dx, back = getattr(binding, name + "_keep8_backward")(dy, codes, scales, rebuild=True, dx=_tensor(torch, np.zeros_like(xp), f32, offset))
    want = _oracle(oracle, name + "_backward", f32, dyp, x8)
    _same(_arrays(torch, dx, f32), want, f32)
    _same(_arrays(torch, back, f32), _oracle(oracle, name, f32, x8), f32)
    alone = getattr(binding, name + "_keep8_backward")(dy, codes, scales)
    _same(_arrays(torch, alone, f32), want, f32)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("n", [1, 5, 8, 127, 128, 129, 255, 511, 513, 1000, 65536, 100003])
def test_sizes(gpu, oracle, name, n):
    _check(gpu, oracle, name, n, n)


@pytest.mark.parametrize("name", NAMES)
def test_special_values(gpu, oracle, name):
    _check(gpu, oracle, name, 5000, 1, special=True)


@pytest.mark.parametrize("name", ["kgelu", "kswish_f32", "kgelu64"])
@pytest.mark.parametrize("offset, code_offset", [(1, 0), (0, 3), (3, 1), (7, 8)])
def test_tensors_off_the_grid(gpu, oracle, name, offset, code_offset):
    _check(gpu, oracle, name, 4099, offset, special=True, offset=offset, code_offset=code_offset)


def test_large_tensors_take_the_streamed_stores(gpu):
    """From 256 MiB of output on; against the same calls on pieces."""
    torch, binding = gpu
    n, piece = (1 << 27) + 1000, 1 << 26
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    x = torch.randn(n, generator=gen, device="cuda").bfloat16()
    y, codes, scales = binding.kgelu_keep8(x)
    dx, back = binding.kgelu_keep8_backward(x, codes, scales, rebuild=True)
    for a in range(0, n, piece):
        part = slice(a, min(n, a + piece))
        groups = slice(a // 128, -(-part.stop // 128))
        y1, c1, s1 = binding.kgelu_keep8(x[part])
        d1, b1 = binding.kgelu_keep8_backward(x[part], c1, s1, rebuild=True)
        for whole, one in ((y, y1), (codes, c1), (dx, d1), (back, b1)):
            assert torch.equal(whole[part], one)
        assert torch.equal(scales[groups], s1)


def test_in_place_empty_and_a_callers_table(gpu, oracle):
    torch, binding = gpu
    xp, dyp = _values(3000, False, 5, False)
    x, dy = _tensor(torch, xp, False), _tensor(torch, dyp, False)
    y, codes, scales = binding.kgelu_keep8(x.clone())
    again, c2, s2 = binding.kgelu_keep8(x, out=x)
    assert again is x and torch.equal(again, y) and torch.equal(c2, codes) and torch.equal(s2, scales)
    dx, back = binding.kgelu_keep8_backward(dy, codes, scales, rebuild=True)
    kept = dy.clone()
    over = binding.kgelu_keep8_backward(kept, codes, scales, dx=kept)
    assert over is kept and torch.equal(over, dx)
    kept = dy.clone()
    d2, b2 = binding.kgelu_keep8_backward(kept, codes, scales, y=kept)
    assert b2 is kept and torch.equal(b2, back) and torch.equal(d2, dx)
    none = torch.empty(0, dtype=torch.bfloat16, device="cuda")
    y, codes, scales = binding.kswish_keep8(none)
    assert y.numel() == codes.numel() == scales.numel() == 0 and binding.kswish_keep8_backward(none, codes, scales).numel() == 0
    table = binding.ktanh_fit_lut_bmin0()
    y, codes, scales = binding.kgelu_keep8(dy, lut=table)
    assert torch.equal(y, binding.kgelu(dy, lut=table))
    x8 = _tensor(torch, _restored(codes.cpu().numpy(), scales.cpu().numpy(), False), False)
    assert torch.equal(binding.kgelu_keep8_backward(dy, codes, scales, lut=table), binding.kgelu_backward(dy, x8, lut=table))


@pytest.mark.parametrize("name, dtype, intervals", [("kgelu", "bfloat16", 32), ("kswish", "bfloat16", 64), ("kgelu", "float32", 64), ("kswish", "float32", 32)])
def test_autograd_keeps_a_byte(gpu, name, dtype, intervals):
    torch, binding = gpu
    from paper_1909_07729_amd import autograd
    torch.manual_seed(0)
    x = torch.randn(33, 257, device="cuda").to(getattr(torch, dtype)).requires_grad_()
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        y = getattr(autograd, name)(x, intervals=intervals, keep=8)
    assert sum(t.numel() * t.element_size() for t in kept) == x.numel() + 4 * -(-x.numel() // 128)
    entry = f"{name}{'64' if intervals == 64 else ''}{'_f32' if dtype == 'float32' else ''}"
    want, codes, scales = getattr(binding, entry + "_keep8")(x.detach())
    assert torch.equal(y, want) and y.shape == x.shape
    dy = torch.randn_like(x)
    assert torch.equal(torch.autograd.grad(y, x, dy, retain_graph=True)[0], getattr(binding, entry + "_keep8_backward")(dy, codes, scales))
    # an expanded gradient, a transposed input, no gradient asked for
    y.sum().backward()
    assert torch.equal(x.grad, getattr(binding, entry + "_keep8_backward")(torch.ones_like(x), codes, scales))
    turned = x.detach().t().requires_grad_()
    assert torch.equal(getattr(autograd, name)(turned, intervals=intervals, keep=8).t(), want)
    with torch.no_grad():
        assert torch.equal(getattr(autograd, name)(x, intervals=intervals, keep=8), want)
    with pytest.raises(ValueError):
        getattr(autograd, name)(x, keep=4)


@pytest.mark.parametrize("name", ["kgelu", "kswish"])
def test_gradient_against_differences(gpu, name):
    """The gradient in Float32 against central differences of the exact activation, |x| <= 2.  Off by: the code, half of 2 / 127 in x where the slope changes
    by at most 0.8 (GELU; Swish 0.5) a unit; K, whose error is at most 0.9e-2 (Table 1 over all inputs), through d slope / dt, at most 0.5 + |x t c (1 + 3 a x^2)|
    <= 0.5 + 2 * 0.97 * 0.798 * 1.54 = 2.9 for GELU, and for Swish 0.5 |1 + x (1 - 2 s)| with t = 2 s - 1, at most 0.5 (1 + 2 * 0.77) = 1.3; the
    differences, 1e-8."""
    torch, binding = gpu
    x = torch.linspace(-2, 2, 4001, dtype=torch.float64)
    exact = (lambda v: torch.nn.functional.gelu(v, approximate="tanh")) if name == "kgelu" else torch.nn.functional.silu
    slope = (exact(x + 1e-4) - exact(x - 1e-4)) / 2e-4
    y, codes, scales = getattr(binding, name + "_f32_keep8")(x.float().cuda())
    got = getattr(binding, name + "_f32_keep8_backward")(torch.ones(4001, device="cuda"), codes, scales).cpu().double()
    bound = 0.8 / 127 + 2.9 * 0.9e-2 if name == "kgelu" else 0.5 / 127 + 1.3 * 0.9e-2
    assert (got - slope).abs().max() < bound + 1e-6


def test_graphs_and_streams(gpu):
    torch, binding = gpu
    from paper_1909_07729_amd import autograd
    torch.manual_seed(0)
    x = torch.randn(70001, device="cuda").bfloat16().requires_grad_()
    dy = torch.randn_like(x)
    eager = autograd.kgelu(x, keep=8)                       # an eager graph of the same leaf lives throughout
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y1, c1, s1 = binding.kgelu_keep8(x.detach())
    torch.cuda.current_stream().wait_stream(side)
    own, c2, s2 = binding.kgelu_keep8(x.detach(), stream=side)
    side.synchronize()
    assert torch.equal(y1, own) and torch.equal(c1, c2) and torch.equal(s1, s2)
    leaf = x.detach().clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, codes, scales = binding.kgelu_keep8(leaf)
        dx, back = binding.kgelu_keep8_backward(dy, codes, scales, rebuild=True)
    for seed in range(3):
        torch.manual_seed(seed)
        leaf.copy_(torch.randn(70001, device="cuda") * 3)
        graph.replay()
        torch.cuda.synchronize()
        want, c, s = binding.kgelu_keep8(leaf)
        d, b = binding.kgelu_keep8_backward(dy, c, s, rebuild=True)
        for got, w in ((y, want), (codes, c), (scales, s), (dx, d), (back, b)):
            assert torch.equal(got, w)
    assert torch.autograd.grad(eager, x, dy)[0].shape == x.shape


def test_both_host_paths_give_the_same(gpu, monkeypatch):
    """Ordinary calls go through C++ where it is built, others through Python."""
    torch, binding = gpu
    from paper_1909_07729_amd import autograd
    assert binding._host is not None
    torch.manual_seed(0)
    for name in NAMES:
        f32 = name.endswith("_f32")
        x = torch.randn(3, 700, device="cuda").to(torch.float32 if f32 else torch.bfloat16)
        table = binding.ktanh_fit_lut64() if "64" in name else binding.ktanh_fit_lut_bmin0()
        results = []
        for host in (binding._host, None):
            monkeypatch.setattr(binding, "_host", host)
            leaf = x.clone().requires_grad_()
            y = getattr(autograd, name.split("64")[0].split("_f32")[0])(leaf, intervals=64 if "64" in name else 32, keep=8)
            made = []
            for lut in (None, table):
                kept = getattr(binding, name + "_keep8")(x, lut=lut)
                made += [*kept, getattr(binding, name + "_keep8_backward")(x, *kept[1:], lut=lut),
                         *getattr(binding, name + "_keep8_backward")(x, *kept[1:], rebuild=True, lut=lut)]
            results.append([y, *torch.autograd.grad(y, leaf, x), *made])
            monkeypatch.undo()
        for a, b in zip(*results):
            assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b), name
    with pytest.raises(binding.KtanhError):
        bad = binding.ktanh_default_lut()
        bad.r[5] = 9
        binding.kgelu_keep8(x.bfloat16(), lut=bad)
    with pytest.raises(TypeError):
        binding.kgelu_keep8(x.double())
    with pytest.raises(ValueError):
        binding.kgelu_keep8_backward(x.bfloat16(), *binding.kgelu_keep8(x[:1].bfloat16())[1:])


def test_one_output_for_both_is_refused(gpu):
    torch, binding = gpu[:2]
    x = torch.randn(1000, device="cuda").bfloat16()
    _, codes, scales = binding.kgelu_keep8(x)
    with pytest.raises(ValueError):
        binding.kgelu_keep8_backward(x, codes, scales, dx=x, y=x)
    with pytest.raises(ValueError):
        both = torch.empty_like(x)
        binding.kgelu_keep8_backward(x, codes, scales, dx=both, y=both)
    dx, y = binding.kgelu_keep8_backward(x, codes, scales, rebuild=True)
    dy = x.clone()
    assert all(torch.equal(a, b) for a, b in zip(binding.kgelu_keep8_backward(dy, codes, scales, dx=dy, y=torch.empty_like(x)), (dx, y)))
    dy = x.clone()
    assert all(torch.equal(a, b) for a, b in zip(binding.kgelu_keep8_backward(dy, codes, scales, dx=torch.empty_like(x), y=dy), (dx, y)))
