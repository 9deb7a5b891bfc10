"""Activations kept in 8 bits where a group holds the type's largest or lowest values, as masked places do: finite values stay finite."""
import numpy as np
import pytest

from test_gpu_keep8 import NAMES, _arrays, _bf16, _checkpoint, _oracle, _restored, _same, _tensor, _wide, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = np.float32(float.fromhex("0x1.020406p121"))


def test_the_largest_scale():
    """Its 127-fold is finite, that of the next one is not."""
    with np.errstate(over="ignore"):
        assert np.isfinite(MOST * np.float32(127)) and np.isinf(np.nextafter(MOST, np.float32(np.inf)) * np.float32(127))


@pytest.mark.parametrize("name", NAMES)
def test_groups_with_the_types_limits(gpu, oracle, name):
    torch, binding = gpu
    f32 = name.endswith("_f32")
    rng = np.random.default_rng(1)
    x = rng.standard_normal(900).astype(np.float32)
    last = np.float32(np.finfo(np.float32).max) if f32 else _wide(np.array([0x7F7F], np.uint16))[0]
    x[5], x[130], x[131], x[256:384] = -last, last, -last, -last
    x[400], x[401] = last, np.inf                       # an infinity beside them
    x[520] = last / 2
    x[640] = np.nextafter(last, np.float32(0)) if f32 else last
    dy = rng.standard_normal(900).astype(np.float32)
    xp, dyp = (x.view(np.uint32), dy.view(np.uint32)) if f32 else (_bf16(x), _bf16(dy))
    values = x if f32 else _wide(xp)
    y, codes, scales = getattr(binding, name + "_keep8")(_tensor(torch, xp, f32))
    _same(_arrays(torch, y, f32), _oracle(oracle, name, f32, xp), f32)
    want_codes, want_scales = _checkpoint(values)
    want_scales = np.minimum(want_scales, MOST)
    assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)
    with np.errstate(over="ignore"):                    # -128, which stands for no value
        x8 = _restored(want_codes, want_scales, f32)
    inside = np.isfinite(values)
    assert np.isfinite(x8.view(np.float32) if f32 else _wide(x8))[inside].all()
    dx, back = getattr(binding, name + "_keep8_backward")(_tensor(torch, dyp, f32), codes, scales, rebuild=True)
    _same(_arrays(torch, dx, f32), _oracle(oracle, name + "_backward", f32, dyp, x8), f32)
    _same(_arrays(torch, back, f32), _oracle(oracle, name, f32, x8), f32)
    if name.startswith("kswish"):       # where the library's own gradient at these values is finite
        assert np.isfinite(dx.cpu().float().numpy()[inside]).all()
