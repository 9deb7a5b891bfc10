"""Calls on activations that keep 8 bits, as they are made of ordinary Python values."""
import numpy as np
import pytest

from test_gpu_keep8 import NAMES, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("host", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_rebuild_is_a_truth_value(gpu, monkeypatch, name, host):
    """The same through C++ and through Python, whatever stands for true."""
    torch, binding = gpu
    if not host:
        monkeypatch.setattr(binding, "_host", None)
    x = torch.randn(2, 700, device="cuda").to(torch.float32 if name.endswith("_f32") else torch.bfloat16)
    _, codes, scales = getattr(binding, name + "_keep8")(x)
    back = getattr(binding, name + "_keep8_backward")
    dx, y = back(x, codes, scales, rebuild=True)
    for yes in (1, np.True_, "output"):
        made = back(x, codes, scales, rebuild=yes)
        assert isinstance(made, tuple) and torch.equal(made[0], dx) and torch.equal(made[1], y)
    for no in (0, np.False_, None, False):
        assert torch.equal(back(x, codes, scales, rebuild=no), dx)
