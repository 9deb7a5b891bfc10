"""Rows and products in 8-bit integers against their definition in 64 bits."""
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


def _rows(x):
    """(codes, scales) of Float32 rows by the definition, in numpy."""
    top = np.abs(x).max(1, keepdims=True, initial=0).astype(np.float32)
    finite = np.isfinite(x).all(1, keepdims=True)
    tiny = top < np.float32(2.0 ** -120)
    with np.errstate(all="ignore"):
        inverse = np.where(tiny, np.float32(0), np.float32(127) / top).astype(np.float32)
        codes = np.where(finite, np.rint(x * inverse), 0).astype(np.int8)
        scales = np.where(tiny, np.float32(0), top / np.float32(127)).astype(np.float32)
    return codes, np.where(finite, scales, np.float32(np.nan))[:, 0]


def _inside(torch, rows, columns, dtype, apart, start):
    """A matrix whose rows are `apart` elements longer than its columns, `start` elements into its memory."""
    room = torch.zeros(rows * (columns + apart) + start + 64, dtype=dtype, device="cuda")
    return room[start:start + rows * (columns + apart)].view(rows, columns + apart)[:, :columns], room


def _x(torch, rows, columns, dtype, seed, apart=0, start=0, special=False):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x, _ = _inside(torch, rows, columns, dtype, apart, start)
    x.copy_(torch.randn((rows, columns), generator=gen, device="cuda") * torch.rand((rows, 1), generator=gen, device="cuda").mul(4).exp())
    if special:
        x[0] = 0
        x[1, columns // 2] = float("nan")
        x[2, -1] = float("inf")
        x[3, 0] = -float("inf")
        x[4] = 2.0 ** -121
        x[5] *= 2.0 ** -110
        x[6] = 3e38
        x[7] = -0.0
    return x


def _activated(torch, binding, x, activation, intervals):
    """The activation by the library's own element-wise call, which has tests of its own."""
    if activation is None:
        return x
    name = f"k{activation}{'64' if intervals == 64 else ''}{'_f32' if x.dtype == torch.float32 else ''}"
    return getattr(binding, name)(x.contiguous())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("columns", [1, 3, 8, 63, 64, 257, 512, 513, 1000, 2048, 4096, 4100, 16384, 16392, 65540, 70001])
@pytest.mark.parametrize("activation, intervals", [(None, 32), ("gelu", 32), ("swish", 64)])
def test_rows(gpu, dtype, columns, activation, intervals):
    torch, binding = gpu
    x = _x(torch, 9, columns, getattr(torch, dtype), columns, special=columns > 2)
    rows = binding.kq8_rows if intervals == 32 else binding.kq8_rows64
    codes, scales = rows(x, activation)
    want, want_scales = _rows(_activated(torch, binding, x, activation, intervals).float().cpu().numpy())
    assert codes.shape == x.shape and codes.stride(0) % 16 == 0
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), want_scales, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("apart, start, codes_apart, codes_start", [(0, 1, 0, 0), (5, 0, 0, 0), (8, 8, 3, 1), (16, 0, 16, 8), (0, 0, 0, 5)])
def test_rows_with_strides(gpu, dtype, apart, start, codes_apart, codes_start):
    torch, binding = gpu
    x = _x(torch, 33, 333, getattr(torch, dtype), 1, apart, start)
    codes, room = _inside(torch, 33, 333, torch.int8, codes_apart, codes_start)
    room.fill_(77)
    got, scales = binding.kq8_rows(x, "gelu", codes=codes)
    assert got is codes
    want, want_scales = _rows(_activated(torch, binding, x, "gelu", 32).float().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), want_scales)
    codes.fill_(77)
    assert (room == 77).all()               # nothing is written between the rows or beside them
    one = x[:1].expand(5, -1)               # the same row five times
    codes, scales = binding.kq8_rows(one)
    assert (codes == codes[0]).all() and (scales == scales[0]).all()


def _codes(torch, rows, columns, seed, apart=0, start=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    codes, room = _inside(torch, rows, columns, torch.int8, apart, start)
    room.copy_(torch.randint(-128, 128, room.shape, generator=gen, device="cuda"))      # also between the rows
    return codes


def _scales(torch, count, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.rand(count, generator=gen, device="cuda") * 1e-3 + 1e-5


def _want(torch, codes, scales, weight, weight_scales, bias, dtype):
    """The definition: the sums exact in 64 bits, then its Float32 operations."""
    sums = codes.double().cpu() @ weight.double().cpu().T
    out = sums.float() * scales.cpu()[:, None] * weight_scales.cpu()
    if bias is not None:
        out = out + bias.cpu()
    return out.to(dtype)


SIZES = [(1, 64, 16), (1, 4096, 4096), (1, 1, 1), (2, 17, 5), (3, 63, 64), (5, 65, 63), (8, 4160, 1000), (16, 1024, 2050), (17, 1024, 513), (32, 2048, 256),
         (33, 100, 1000), (63, 640, 190), (64, 4096, 1024), (65, 128, 65), (100, 1001, 2003), (127, 16384, 128), (128, 512, 257), (255, 1000, 255),
         (256, 256, 256), (257, 4096, 512), (300, 129, 777), (513, 2048, 1025), (1000, 1024, 1000), (1024, 16, 512), (2048, 4096, 768)]


@pytest.mark.parametrize("rows, inner, outer", SIZES)
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_products(gpu, rows, inner, outer, dtype):
    """Identical bits: every operation of the definition is exact or rounded once."""
    torch, binding = gpu
    pad = -inner % 16
    codes, weight = _codes(torch, rows, inner, 1, pad), _codes(torch, outer, inner, 2, pad)
    scales, weight_scales = _scales(torch, rows, 3), _scales(torch, outer, 4)
    bias = _scales(torch, outer, 5) * 1e3 if rows % 2 else None
    out = binding.kq8_product(codes, scales, weight, weight_scales, bias, out_dtype=getattr(torch, dtype))
    assert torch.equal(out.cpu(), _want(torch, codes, scales, weight, weight_scales, bias, out.dtype))


# Every kind of tile with ends of rows, channels and inner dimension that fill none, in one part and in several (tests/test_q8_plans.py holds the plans to these).
TILES = [(8190, 1040, 8190), (2040, 520, 6130), (2040, 1160, 4090), (1000, 656, 4000), (770, 1040, 2000), (900, 8200, 900), (24, 528, 50000), (30, 300, 30000),
         (500, 16400, 1000), (100, 16400, 500), (1000, 131071, 70)]


@pytest.mark.parametrize("rows, inner, outer", TILES)
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_products_in_tiles(gpu, rows, inner, outer, dtype):
    torch, binding = gpu
    pad = -inner % 16
    codes, weight = _codes(torch, rows, inner, 1, pad), _codes(torch, outer, inner, 2, pad)
    scales, weight_scales = _scales(torch, rows, 3), _scales(torch, outer, 4)
    room = torch.full((rows + 1, outer + 3), 7.0, dtype=getattr(torch, dtype), device="cuda")
    out = binding.kq8_product(codes, scales, weight, weight_scales, out=room[:rows, :outer])
    assert torch.equal(out.cpu(), _want(torch, codes, scales, weight, weight_scales, None, out.dtype))
    assert (room[rows] == 7).all() and (room[:, outer:] == 7).all()


@pytest.mark.parametrize("rows, inner, outer", [(1, 1000, 100), (16, 129, 70), (40, 333, 200), (130, 1000, 131), (300, 777, 301)])
@pytest.mark.parametrize("layout", range(6))
def test_products_with_strides(gpu, rows, inner, outer, layout):
    torch, binding = gpu
    x_apart, x_start, w_apart, w_start, out_apart, out_start = [(0, 0, 0, 0, 0, 0), (1, 0, 0, 3, 1, 1), (7, 16, 16, 0, 0, 2), (24, 8, 40, 24, 3, 0),
                                                               (-inner % 16, 0, -inner % 16, 0, 5, 4), (-inner % 16 + 16, 1, -inner % 16, 0, 64, 0)][layout]
    codes, weight = _codes(torch, rows, inner, 1, x_apart, x_start), _codes(torch, outer, inner, 2, w_apart, w_start)
    scales, weight_scales, bias = _scales(torch, rows, 3), _scales(torch, outer, 4), _scales(torch, outer, 5)
    for dtype in (torch.bfloat16, torch.float32):
        out, room = _inside(torch, rows, outer, dtype, out_apart, out_start)
        room.fill_(7)
        got = binding.kq8_product(codes, scales, weight, weight_scales, bias, out=out)
        assert got is out
        assert torch.equal(out.cpu(), _want(torch, codes, scales, weight, weight_scales, bias, dtype))
        out.fill_(7)
        assert (room == 7).all()


def test_the_largest_sums_are_exact(gpu):
    torch, binding = gpu
    inner = 131071
    codes = torch.full((2, inner + 1), -128, dtype=torch.int8, device="cuda")[:, :inner]
    weight = torch.full((20, inner + 1), -128, dtype=torch.int8, device="cuda")[:, :inner]
    weight[1::2] = 127
    one = torch.ones(20, device="cuda")
    out = binding.kq8_product(codes, one[:2], weight, one, out_dtype=torch.float32)
    want = torch.tensor([128 * 128 * inner, -128 * 127 * inner], dtype=torch.float64).float().repeat(10)
    assert torch.equal(out.cpu(), want.expand(2, -1))
    with pytest.raises(binding.KtanhError):
        binding.kq8_product(*(torch.zeros(s, device="cuda", dtype=t) for s, t in (((1, 131072), torch.int8), ((1,), torch.float32), ((1, 131072), torch.int8),
                                                                                 ((1,), torch.float32))))


@pytest.mark.parametrize("rows, inner, outer", [(1, 256, 300), (1, 4096, 512), (2, 1001, 77), (4, 16384, 64), (7, 512, 512), (16, 1000, 260), (40, 256, 128),
                                                (200, 1024, 512)])
@pytest.mark.parametrize("dtype, activation, intervals", [("bfloat16", None, 32), ("bfloat16", "gelu", 32), ("float32", "swish", 64), ("float32", None, 32),
                                                          ("bfloat16", "swish", 64), ("float32", "gelu", 32)])
def test_linear_is_rows_and_product(gpu, rows, inner, outer, dtype, activation, intervals):
    torch, binding = gpu
    special = rows >= 8 and inner > 2
    x = _x(torch, rows, inner, getattr(torch, dtype), rows, apart=rows % 3, special=special)
    weight, weight_scales = binding.kq8_rows(_x(torch, outer, inner, torch.float32, 9))
    bias = _scales(torch, outer, 5) if rows % 2 else None
    linear, to_rows = (binding.kq8_linear, binding.kq8_rows) if intervals == 32 else (binding.kq8_linear64, binding.kq8_rows64)
    codes, scales = to_rows(x, activation)
    for out_dtype in (torch.bfloat16, torch.float32):
        out = linear(x, weight, weight_scales, bias, activation=activation, out_dtype=out_dtype)
        want = _want(torch, codes, scales, weight, weight_scales, bias, out_dtype)
        bad = want.isnan()
        assert torch.equal(out.cpu().isnan(), bad) and torch.equal(out.cpu()[~bad], want[~bad])
        assert bad.any(1).tolist() == [special and activation is None and i in (1, 2, 3) or special and bool(codes[i].eq(0).all() and scales[i].isnan())
                                       for i in range(rows)]


def test_how_far_the_product_is_from_float(gpu):
    """Against the product of the unrounded values in 64 bits.  A code is off by at most half a step: the sum over i of |w| scale / 2 + |x| w_scale / 2 +
    scale w_scale / 4, and what Float32 and BFloat16 round: 2^-8 of the result."""
    torch, binding = gpu
    x, w = _x(torch, 50, 1000, torch.bfloat16, 1), _x(torch, 300, 1000, torch.float32, 2)
    weight, weight_scales = binding.kq8_rows(w)
    codes, scales = binding.kq8_rows(x)
    out = binding.kq8_linear(x, weight, weight_scales).double()
    a, b, s, t = x.double(), w.double(), scales.double()[:, None], weight_scales.double()
    bound = s / 2 * b.abs().sum(1) + a.abs().sum(1, keepdim=True) * t / 2 + 1000 * s * t / 4
    want = a @ b.T
    assert ((out - want).abs() <= bound * (1 + 2.0 ** -7) + want.abs() * 2.0 ** -8).all()


def test_empty_calls(gpu):
    torch, binding = gpu
    weight, weight_scales = _codes(torch, 6, 32, 1), _scales(torch, 6, 2)
    assert binding.kq8_linear(torch.empty((0, 32), device="cuda"), weight, weight_scales).shape == (0, 6)
    assert binding.kq8_linear(torch.ones((3, 32), device="cuda"), weight[:0], weight_scales[:0]).shape == (3, 0)
    bias = _scales(torch, 6, 3)
    nothing = binding.kq8_linear(torch.empty((3, 0), device="cuda"), weight[:, :0], weight_scales, bias, out_dtype=torch.float32)
    assert torch.equal(nothing, bias.expand(3, -1))
    codes, scales = binding.kq8_rows(torch.empty((3, 0), device="cuda"))
    assert codes.shape == (3, 0) and (scales == 0).all()
    assert binding.kq8_rows(torch.empty((0, 9), device="cuda"))[0].shape == (0, 9)


def test_graphs_streams_and_repeated_calls(gpu):
    torch, binding = gpu
    x = _x(torch, 4, 512, torch.bfloat16, 1)
    weight, weight_scales = binding.kq8_rows(_x(torch, 320, 512, torch.bfloat16, 2))
    wide, wide_scales = binding.kq8_rows(_x(torch, 512, 320, torch.bfloat16, 3))

    def both(rows, stream=None):
        h = binding.kq8_linear(rows, weight, weight_scales, stream=stream)
        return binding.kq8_linear(h, wide, wide_scales, activation="gelu", stream=stream)
    graphs = []
    for _ in range(2):                      # two graphs, each with workspaces of its own pool
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both(x)
        graphs.append((graph, out))
    for seed in range(3):
        x.copy_(_x(torch, 4, 512, torch.bfloat16, 10 + seed))
        want = both(x)
        for graph, out in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one = both(x)
    two = both(x, stream=side)
    side.synchronize()
    assert torch.equal(one, want) and torch.equal(two, want)


def test_both_host_paths_give_the_same(gpu, monkeypatch):
    """Ordinary calls go through C++ where it is built, others through Python."""
    torch, binding = gpu
    assert binding._host is not None
    x = _x(torch, 5, 100, torch.bfloat16, 1, apart=3)
    weight, weight_scales = binding.kq8_rows(_x(torch, 70, 100, torch.bfloat16, 2))
    codes, scales = binding.kq8_rows(x)
    bias, table = _scales(torch, 70, 3), binding.ktanh_fit_lut_bmin0()
    wide = torch.empty((5, 90), dtype=torch.float32, device="cuda")
    results = []
    for host in (binding._host, None):
        monkeypatch.setattr(binding, "_host", host)
        made = [binding.kq8_linear(v, weight, weight_scales, b, activation=act, out_dtype=dtype)
                for v in (x, x.float()) for b in (None, bias) for act in (None, "gelu", "swish") for dtype in (torch.bfloat16, torch.float32)]
        made += [binding.kq8_linear64(x, weight, weight_scales, activation="gelu"), binding.kq8_linear(x, weight, weight_scales, activation="gelu", lut=table),
                 binding.kq8_product(codes, scales, weight, weight_scales, bias), binding.kq8_product(codes, scales, weight, weight_scales, out_dtype=torch.float32),
                 binding.kq8_linear(x, weight, weight_scales, out=wide[:, :70]).clone(), binding.kq8_product(codes, scales, weight, weight_scales, out=wide[:, 20:]).clone()]
        results.append(made)
        monkeypatch.undo()
    for a, b in zip(*results):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_refused_calls(gpu):
    torch, binding = gpu
    x, w, one = torch.ones((4, 64), device="cuda"), torch.ones((8, 64), dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
    for call, error in ((lambda: binding.kq8_linear(x, w[:, :32], one), ValueError), (lambda: binding.kq8_linear(x, w, one[:4]), ValueError),
                        (lambda: binding.kq8_linear(x, w.short(), one), TypeError), (lambda: binding.kq8_linear(x.half(), w, one), TypeError),
                        (lambda: binding.kq8_linear(x, w, one, out_dtype=torch.float16), TypeError), (lambda: binding.kq8_linear(x, w, one, one.double()), TypeError),
                        (lambda: binding.kq8_linear(x, w, one, activation="relu"), ValueError), (lambda: binding.kq8_linear(x.t(), w[:, :4], one), ValueError),
                        (lambda: binding.kq8_linear(x, w, one, out=torch.empty((4, 9), device="cuda")), ValueError),
                        (lambda: binding.kq8_linear(x, w, one, out=torch.empty(8, device="cuda").expand(4, 8)), ValueError),
                        (lambda: binding.kq8_rows(x[0]), ValueError), (lambda: binding.kq8_rows(x, codes=w), ValueError),
                        (lambda: binding.kq8_rows(x, codes=w[:1].expand(4, 64)), ValueError), (lambda: binding.kq8_product(w, one[:2], w, one), ValueError)):
        with pytest.raises(error):
            call()
