"""Products in 8-bit integers through the blocks of 64 by 64 whose wavefronts share the inner dimension: operands off the 16-byte grid, or rows too far apart for
tiles.  Identical bits."""
import pytest

from test_gpu_q8 import _codes, _inside, _scales, _want, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

# rows, inner, outer; codes: apart, start; weights: apart, start (tests/test_q8_ways.py holds these to their kernel)
OFF_GRID = [(777, 1001, 2003, 0, 0, 0, 0), (513, 333, 1025, 2, 1, 5, 3), (2000, 200, 5000, 1, 0, 8, 8), (1000, 640, 700, 0, 0, 0, 1), (100, 4097, 3000, 0, 7, 0, 0),
            (3000, 15, 300, 0, 0, 0, 0), (700, 64, 500, 16, 5, 0, 0), (70, 20000, 2100, 0, 0, 3, 0)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("case", OFF_GRID)
def test_off_the_grid(gpu, case, dtype):
    torch, binding = gpu
    rows, inner, outer, x_apart, x_start, w_apart, w_start = case
    codes, weight = _codes(torch, rows, inner, 1, x_apart, x_start), _codes(torch, outer, inner, 2, w_apart, w_start)
    scales, weight_scales, bias = _scales(torch, rows, 3), _scales(torch, outer, 4), _scales(torch, outer, 5) if rows % 2 else None
    out, room = _inside(torch, rows, outer, getattr(torch, dtype), rows % 5, rows % 3)
    room.fill_(7)
    binding.kq8_product(codes, scales, weight, weight_scales, bias, out=out)
    assert torch.equal(out.cpu(), _want(torch, codes, scales, weight, weight_scales, bias, out.dtype))
    out.fill_(7)
    assert (room == 7).all()


# rows, inner, outer, step of the codes' rows, step of the weights'
FAR = [(50, 200, 2800, 1 << 23, 208), (300, 1040, 500, 1056, 1 << 23), (64, 77, 2100, (1 << 23) + 16, 80)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows, inner, outer, x_step, w_step", FAR)
def test_far_rows_on_the_grid(gpu, rows, inner, outer, x_step, w_step, dtype):
    torch, binding = gpu

    def apart(t, step):
        room = torch.full(((len(t) - 1) * step + t.shape[1],), 99, dtype=torch.int8, device="cuda")
        far = room.as_strided(t.shape, (step, 1))
        far.copy_(t)
        return far
    codes, weight = _codes(torch, rows, inner, 1), _codes(torch, outer, inner, 2)
    scales, weight_scales, bias = _scales(torch, rows, 3), _scales(torch, outer, 4), _scales(torch, outer, 5)
    out = binding.kq8_product(apart(codes, x_step), scales, apart(weight, w_step), weight_scales, bias, out_dtype=getattr(torch, dtype))
    assert torch.equal(out.cpu(), _want(torch, codes, scales, weight, weight_scales, bias, out.dtype))


def test_weights_off_the_grid_through_linear(gpu):
    """The rows of codes that the call makes are on the grid, the weights are not."""
    torch, binding = gpu
    x = torch.randn((600, 1001), generator=torch.Generator("cuda").manual_seed(6), device="cuda").bfloat16()
    weight, weight_scales = _codes(torch, 1000, 1001, 2), _scales(torch, 1000, 4)
    codes, scales = binding.kq8_rows(x, "gelu")
    out = binding.kq8_linear(x, weight, weight_scales, activation="gelu", out_dtype=torch.float32)
    assert torch.equal(out.cpu(), _want(torch, codes, scales, weight, weight_scales, None, torch.float32))
