"""Host-side checks of the choice of a token, that need no GPU: what is refused, before anything is launched."""
import ctypes
import os
import subprocess

import pytest
import torch

from conftest import ROOT


@pytest.fixture(scope="module")
def binding():
    from paper_1909_07729_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        from paper_1909_07729_amd import build
        build.build_library()
    b.load_library()
    return b


NULL, FAKE = ctypes.c_void_p(0), ctypes.c_void_p(0x1000)     # never dereferenced: rejected on the host


def _shape(binding, **changes):
    values = dict(rows=4, vocabulary=1000, row=1000, f32=0, cap=0.0, temperature=1.0, top_p=1.0, min_p=0.0, top_k=0)
    return binding.KsampleShape(**{**values, **changes})


def test_the_structure_has_the_headers_layout(binding, tmp_path):
    source, exe = tmp_path / "layout.c", tmp_path / "layout"
    fields = [n for n, _ in binding.KsampleShape._fields_]
    source.write_text('#include <stdio.h>\n#include "ktanh.h"\nint main(void) {\n' +
                      "".join(f'printf("%zu\\n", offsetof(ksample_shape_t, {n}));\n' for n in fields) +
                      'printf("%zu\\n", sizeof(ksample_shape_t));\nreturn 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [getattr(binding.KsampleShape, n).offset for n in fields] + [ctypes.sizeof(binding.KsampleShape)]


def test_entry_points_refuse(binding):
    lib, nan = binding.load_library(), float("nan")
    for name, table in (("ksample", binding.ktanh_default_lut()), ("ksample64", binding.ktanh_fit_lut64())):
        def call(shape, logits=FAKE, uniform=FAKE, temperature=NULL, top_k=NULL, top_p=NULL, min_p=NULL, tokens=FAKE, workspace=FAKE, lut=None):
            return getattr(lib, name)(shape, logits, uniform, temperature, top_k, top_p, min_p, tokens, workspace, lut, NULL)
        assert call(None) == 1 and call(_shape(binding, rows=0), NULL, NULL, tokens=NULL) == 0
        for missing in ("logits", "uniform", "tokens"):
            assert call(_shape(binding), **{missing: NULL}) == 1
        for bad in (dict(vocabulary=0), dict(vocabulary=1 << 20), dict(rows=(1 << 24) + 1), dict(rows=1 << 22), dict(rows=1 << 21, vocabulary=40000), dict(row=(1 << 40) + 1), dict(temperature=-1.0), dict(temperature=nan),
                    dict(temperature=float("inf")), dict(top_p=1.5), dict(top_p=nan), dict(top_p=-0.1), dict(min_p=1.5), dict(min_p=nan), dict(cap=-1.0),
                    dict(cap=nan), dict(cap=float("inf")), dict(cap=1e-31)):
            assert call(_shape(binding, **bad)) == 4, bad
        assert call(_shape(binding), logits=ctypes.c_void_p(0x1001)) == 2 and call(_shape(binding, f32=1), logits=ctypes.c_void_p(0x1002)) == 2
        for off in ("uniform", "temperature", "top_k", "top_p", "min_p"):
            assert call(_shape(binding), **{off: ctypes.c_void_p(0x1002)}) == 2
        assert call(_shape(binding), tokens=ctypes.c_void_p(0x1004)) == 2 and call(_shape(binding), workspace=ctypes.c_void_p(0x1008)) == 2
        assert call(_shape(binding, vocabulary=32769), workspace=NULL) == 1
        table.r[5] = 9
        assert call(_shape(binding, cap=30.0), lut=table) == 3


def test_workspace(binding):
    size = binding.load_library().ksample_workspace
    assert size(_shape(binding, vocabulary=32768)) == 0 and size(_shape(binding, rows=0, vocabulary=40000)) == 0
    assert size(_shape(binding, vocabulary=32769)) == 4 * 5 * (1024 * 8 + 20) + 4 * (2048 * 8 + 8)


def test_binding_refuses(binding):
    with pytest.raises(ValueError):
        binding.ksample(torch.zeros(4, 100), torch.zeros(4))            # host memory
