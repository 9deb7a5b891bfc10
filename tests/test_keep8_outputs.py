"""One memory for both outputs of a gradient from 8 bits is refused by the library, before anything is launched."""
import ctypes

import pytest

from test_keep8_boundary import NAMES, NULL, binding  # noqa: F401

DY, CODES, SCALES, DX = (ctypes.c_void_p(i << 20) for i in range(1, 5))         # never dereferenced: refused on the host


@pytest.mark.parametrize("name", NAMES)
def test_one_memory_for_both_outputs(binding, name):
    back = getattr(binding.load_library(), name + "_backward")
    assert back(DY, CODES, SCALES, DX, DX, 100, None, NULL) == 4
    assert back(DY, CODES, SCALES, DY, DY, 100, None, NULL) == 4
    assert back(DY, CODES, SCALES, DX, DX, 0, None, NULL) == 0
