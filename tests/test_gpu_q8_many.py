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
