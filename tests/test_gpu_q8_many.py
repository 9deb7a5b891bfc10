"""Rows and products in 8-bit integers of more rows or channels than one launch has lanes for, against the same calls on fewer."""
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


@pytest.mark.parametrize("rows, inner", [((1 << 26) + 5, 4), ((1 << 26) - 1, 3), ((1 << 25) + 3, 520)])
def test_rows(gpu, rows, inner):
    """From 2^26 rows on where a row has a wavefront, from 2^25 where it has two."""
    torch, binding = gpu
    gen = torch.Generator("cuda").manual_seed(1)
    if inner < 64:
        x = torch.randn((rows, inner), generator=gen, device="cuda").bfloat16()
    else:       # every row the same memory
        x = torch.randn((1, inner), generator=gen, device="cuda").bfloat16().expand(rows, -1)
    codes, scales = torch.full((rows, inner), 99, dtype=torch.int8, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    binding.kq8_rows(x, "gelu", codes=codes, scales=scales)
    part = 1 << 24
    for at in range(0, rows, part):
        end = min(at + part, rows)
        if inner < 64:
            want = binding.kq8_rows(x[at:end], "gelu")
            assert torch.equal(codes[at:end], want[0]) and torch.equal(scales[at:end], want[1])
        else:
            want = binding.kq8_rows(x[:1], "gelu")
            assert (codes[at:end] == want[0]).all() and (scales[at:end] == want[1]).all()


# rows, inner, outer, whether on the 16-byte grid: tests/test_q8_ways.py holds these to more than one launch
PRODUCTS = [(5000000, 17, 1, 0), (4200000, 17, 70, 0), (1, 17, (1 << 27) + 100, 0), (1 << 30, 16, 1, 1)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows, inner, outer, aligned", PRODUCTS)
def test_products(gpu, rows, inner, outer, aligned, dtype):
    """Against the definition, a part of the results at a time: exact sums, Float32 operations."""
    torch, binding = gpu
    gen = torch.Generator("cuda").manual_seed(2)

    def operand(count):     # many channels, or very many rows, are the same memory
        same = count > 1 << 24
        room = torch.randint(-128, 128, (16 + (1 if same else count) * inner,), generator=gen, dtype=torch.int8, device="cuda")
        t = room[0 if aligned else 1:][:(1 if same else count) * inner].view(-1, inner)
        return t.expand(count, -1) if same else t
    codes, weight = operand(rows), operand(outer)
    scales, weight_scales, bias = (torch.rand(n, generator=gen, device="cuda") + 0.5 for n in (rows, outer, outer))
    out = torch.full((rows, outer), 7.0, dtype=getattr(torch, dtype), device="cuda")
    binding.kq8_product(codes, scales, weight, weight_scales, bias, out=out)
    part = max(1, (1 << 24) // max(1, min(outer, 1 << 20)))
    channels = 1 << 24
    for t in range(0, rows, part):
        for o in range(0, outer, channels):
            rows_here, channels_here = slice(t, min(t + part, rows)), slice(o, min(o + channels, outer))
            sums = codes[rows_here].float() @ weight[channels_here].float().t()         # below 2^24: exact in Float32
            want = sums * scales[rows_here, None] * weight_scales[channels_here] + bias[channels_here]
            assert torch.equal(out[rows_here, channels_here], want.to(out.dtype)), (t, o)


def test_linear(gpu):
    torch, binding = gpu
    rows, inner, outer = (1 << 26) + 5, 4, 2
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn((rows, inner), generator=gen, device="cuda").bfloat16()
    weight = torch.randint(-128, 128, (outer, inner), generator=gen, dtype=torch.int8, device="cuda")
    weight_scales = torch.rand(outer, generator=gen, device="cuda")
    out = binding.kq8_linear(x, weight, weight_scales, activation="swish")
    for t in range(0, rows, 1 << 22):
        assert torch.equal(out[t:t + (1 << 22)], binding.kq8_linear(x[t:t + (1 << 22)], weight, weight_scales, activation="swish"))
