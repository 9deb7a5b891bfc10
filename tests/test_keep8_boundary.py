"""Host-side checks of the activations that keep 8 bits, that need no GPU: what is refused, before anything is launched."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    from paper_1909_07729_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        from paper_1909_07729_amd import build
        build.build_library()
    b.load_library()
    return b


NULL, FAKE = ctypes.c_void_p(0), ctypes.c_void_p(0x1000)     # never dereferenced: rejected on the host
NAMES = [f"k{a}{w}{t}_keep8" for a in ("swish", "gelu") for w in ("", "64") for t in ("", "_f32")]


@pytest.mark.parametrize("name", NAMES)
def test_entry_points_refuse(binding, name):
    lib = binding.load_library()
    size = 4 if "_f32" in name else 2
    most = (2 ** 26 - 1) * 64 * (16 // size)
    forward, backward = getattr(lib, name), getattr(lib, name + "_backward")

    def out(n=100, x=FAKE, y=FAKE, codes=FAKE, scales=FAKE, lut=None):
        return forward(x, y, codes, scales, n, lut, NULL)

    def back(n=100, dy=FAKE, codes=FAKE, scales=FAKE, dx=FAKE, y=FAKE, lut=None):
        return backward(dy, codes, scales, dx, y, n, lut, NULL)
    assert out(0, NULL, NULL, NULL, NULL) == 0 and back(0, NULL, NULL, NULL, NULL, NULL) == 0
    for missing in ("x", "y", "codes", "scales"):
        assert out(**{missing: NULL}) == 1, missing
    for missing in ("dy", "codes", "scales", "dx"):
        assert back(**{missing: NULL}) == 1, missing
    off, odd = ctypes.c_void_p(0x1000 + size // 2), ctypes.c_void_p(0x1002)
    for bad in ("x", "y"):
        assert out(**{bad: off}) == 2
    for bad in ("dy", "dx", "y"):
        assert back(**{bad: off}) == 2
    assert out(scales=odd) == 2 and back(scales=odd) == 2
    assert out(most + 1) == 4 and back(most + 1) == 4
    table = binding.ktanh_fit_lut64() if "64" in name else binding.ktanh_default_lut()
    table.r[5] = 9
    assert out(lut=table) == 3 and back(lut=table) == 3


def test_binding_and_autograd_refuse(binding):
    from paper_1909_07729_amd import autograd
    x = torch.zeros(256, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.kgelu_keep8(x)                              # host memory
    with pytest.raises(ValueError):
        binding.kgelu_keep8_backward(x, torch.zeros(256, dtype=torch.int8), torch.zeros(2))
    with pytest.raises(ValueError):
        autograd.kgelu(x, keep=4)
    with pytest.raises(ValueError):
        autograd.kswish(x, keep=16)
    with pytest.raises(ValueError):
        autograd.kgelu(x, intervals=48, keep=8)
