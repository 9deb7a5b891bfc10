"""Offsets past 32 bits: tensors of more than 2^32 values, and rows further apart than that."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1909_07729_amd import binding
    torch.cuda.set_device(0)
    yield torch, binding
    torch.cuda.empty_cache()


def test_checkpoints(gpu):
    torch, binding = gpu
    n, part = (1 << 32) + 1280 + 5, 1 << 20
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator("cuda").manual_seed(1)
    places = [0, (1 << 31) - part, (1 << 32) - part // 2, n - (n % 128) - 256]       # whole groups from each on
    for at in places:
        x[at:at + part] = torch.randn(min(part, n - at), generator=gen, device="cuda").bfloat16()
    y, codes, scales = binding.kgelu_keep8(x)
    dx = binding.kgelu_keep8_backward(x, codes, scales)
    for at in places:
        end = min(at + part, n)
        want = binding.kgelu_keep8(x[at:end].clone())
        assert torch.equal(y[at:end], want[0]) and torch.equal(codes[at:end], want[1]) and torch.equal(scales[at // 128:-(-end // 128)], want[2])
        assert torch.equal(dx[at:end], binding.kgelu_keep8_backward(x[at:end].clone(), want[1], want[2]))


def _apart(torch, rows, columns, step, dtype):
    room = torch.empty((rows - 1) * step + columns, dtype=dtype, device="cuda")
    return room.as_strided((rows, columns), (step, 1))


@pytest.mark.parametrize("rows", [3, 40])
def test_products(gpu, rows):
    """Rows of values, codes, weights and results each more than 2^31 bytes from the first to the last."""
    torch, binding = gpu
    step, inner, outer = (1 << 32) // (rows - 1) // 16 * 16, 320, 50
    gen = torch.Generator("cuda").manual_seed(2)
    x, codes, out = (_apart(torch, rows, c, step, t) for c, t in ((inner, torch.bfloat16), (inner, torch.int8), (outer, torch.float32)))
    weight = _apart(torch, outer, inner, (1 << 32) // 49 // 16 * 16, torch.int8)
    x.copy_(torch.randn((rows, inner), generator=gen, device="cuda"))
    weight.copy_(torch.randint(-127, 128, (outer, inner), generator=gen, device="cuda"))
    near, scales = weight.contiguous(), torch.rand(outer, generator=gen, device="cuda")
    assert codes.stride(0) == x.stride(0) == out.stride(0) == step
    _, row_scales = binding.kq8_rows(x, "gelu", codes=codes)
    want_codes, want_scales = binding.kq8_rows(x.contiguous(), "gelu")
    assert torch.equal(codes, want_codes) and torch.equal(row_scales, want_scales)
    want = binding.kq8_product(want_codes, want_scales, near, scales, out_dtype=torch.float32)
    assert torch.equal(binding.kq8_product(codes, row_scales, weight, scales, out=out), want)
    out.zero_()
    assert torch.equal(binding.kq8_linear(x, weight, scales, activation="gelu", out=out), want)


@pytest.mark.parametrize("vocabulary", [5000, 40000])
def test_tokens(gpu, vocabulary):
    torch, binding = gpu
    gen = torch.Generator("cuda").manual_seed(3)
    logits = _apart(torch, 4, vocabulary, (1 << 31) + 3, torch.bfloat16)
    logits.copy_(torch.randn((4, vocabulary), generator=gen, device="cuda") * 3)
    u = torch.rand(4, generator=gen, device="cuda")
    for settings in (dict(top_p=0.9), dict(top_k=30), dict(temperature=0.0)):
        assert torch.equal(binding.ksample(logits, u, **settings), binding.ksample(logits.contiguous(), u, **settings))
