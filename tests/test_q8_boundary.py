"""Host-side checks of rows and products in 8-bit integers, that need no GPU: what is refused, before anything is launched."""
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
ODD = ctypes.c_void_p(0x1001)


def _shape(binding, **changes):
    values = dict(rows=8, inner=64, outer=32, x_row=64, w_row=64, out_row=32, x_f32=0, out_f32=0, activation=0)
    return binding.Kq8Shape(**{**values, **changes})


def test_the_structure_has_the_headers_layout(binding, tmp_path):
    source, exe = tmp_path / "layout.c", tmp_path / "layout"
    fields = [n for n, _ in binding.Kq8Shape._fields_]
    source.write_text('#include <stdio.h>\n#include "ktanh.h"\nint main(void) {\n' +
                      "".join(f'printf("%zu\\n", offsetof(kq8_shape_t, {n}));\n' for n in fields) +
                      'printf("%zu %d %d %d\\n", sizeof(kq8_shape_t), KQ8_NONE, KQ8_SWISH, KQ8_GELU);\nreturn 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    codes = [binding._ACTIVATIONS[a] for a in (None, "swish", "gelu")]
    assert [int(v) for v in out] == [getattr(binding.Kq8Shape, n).offset for n in fields] + [ctypes.sizeof(binding.Kq8Shape), *codes]


def test_rows_refuse(binding):
    lib = binding.load_library()
    for name, table in (("kq8_rows", binding.ktanh_default_lut()), ("kq8_rows64", binding.ktanh_fit_lut64())):
        def call(shape, x=FAKE, codes=FAKE, codes_row=64, scales=FAKE, lut=None):
            return getattr(lib, name)(shape, x, codes, codes_row, scales, lut, NULL)
        assert call(None) == 1 and call(_shape(binding, rows=0), NULL, NULL, 64, NULL) == 0
        for missing in ("x", "codes", "scales"):
            assert call(_shape(binding), **{missing: NULL}) == 1
        assert call(_shape(binding), x=ODD) == 2 and call(_shape(binding, x_f32=1), x=ctypes.c_void_p(0x1002)) == 2
        assert call(_shape(binding), scales=ctypes.c_void_p(0x1002)) == 2
        for bad in (dict(activation=3), dict(activation=-1), dict(rows=(1 << 30) + 1), dict(inner=(1 << 30) + 1), dict(x_row=(1 << 40) + 1)):
            assert call(_shape(binding, **bad)) == 4, bad
        assert call(_shape(binding), codes_row=63) == 4 and call(_shape(binding), codes_row=(1 << 40) + 1) == 4
        table.r[5] = 9
        assert call(_shape(binding, activation=2), lut=table) == 3


def test_products_refuse(binding):
    lib = binding.load_library()

    def product(shape, codes=FAKE, scales=FAKE, w=FAKE, w_scale=FAKE, bias=NULL, out=FAKE, workspace=FAKE):
        return lib.kq8_product(shape, codes, scales, w, w_scale, bias, out, workspace, NULL)

    def linear(shape, x=FAKE, w=FAKE, w_scale=FAKE, bias=NULL, out=FAKE, workspace=FAKE, lut=None):
        return lib.kq8_linear(shape, x, w, w_scale, bias, out, workspace, lut, NULL)

    def linear64(shape, x=FAKE, w=FAKE, w_scale=FAKE, bias=NULL, out=FAKE, workspace=FAKE, lut=None):
        return lib.kq8_linear64(shape, x, w, w_scale, bias, out, workspace, lut, NULL)
    for call, needed in ((product, ("codes", "scales", "w", "w_scale", "out")), (linear, ("x", "w", "w_scale", "out", "workspace")),
                         (linear64, ("x", "w", "w_scale", "out", "workspace"))):
        assert call(None) == 1
        assert call(_shape(binding, rows=0), **dict.fromkeys(needed, NULL)) == 0 and call(_shape(binding, outer=0), **dict.fromkeys(needed, NULL)) == 0
        for missing in needed:
            assert call(_shape(binding), **{missing: NULL}) == 1, missing
        for bad in (dict(inner=131072), dict(rows=(1 << 30) + 1), dict(outer=(1 << 30) + 1), dict(out_row=31), dict(w_row=(1 << 40) + 1),
                    dict(x_row=(1 << 40) + 1), dict(out_row=(1 << 40) + 1)):
            assert call(_shape(binding, **bad)) == 4, bad
        half = ctypes.c_void_p(0x1002)
        assert call(_shape(binding), w_scale=half) == 2 and call(_shape(binding), bias=half) == 2
        assert call(_shape(binding), out=ODD) == 2 and call(_shape(binding, out_f32=1), out=half) == 2
    assert product(_shape(binding), scales=ctypes.c_void_p(0x1002)) == 2 and product(_shape(binding), workspace=ctypes.c_void_p(0x1008)) == 2
    parts = _shape(binding, rows=64, inner=16384, outer=1024, x_row=16384, w_row=16384, out_row=1024)
    assert lib.kq8_product_workspace(parts) > 0 and product(parts, workspace=NULL) == 1
    assert linear(_shape(binding), x=ODD) == 2 and linear(_shape(binding), workspace=ctypes.c_void_p(0x1008)) == 2
    assert linear(_shape(binding, activation=7)) == 4
    table = binding.ktanh_default_lut()
    table.r[5] = 9
    assert linear(_shape(binding, activation=1), lut=table) == 3


def test_workspace(binding):
    lib = binding.load_library()
    assert lib.kq8_linear_workspace(_shape(binding)) == 8 * (64 + 4)
    assert lib.kq8_linear_workspace(_shape(binding, inner=65)) == 8 * (80 + 4)
    few = _shape(binding, rows=64, inner=16384, outer=1024, x_row=16384, w_row=16384, out_row=1024)
    assert lib.kq8_linear_workspace(few) == 64 * (16384 + 4) + lib.kq8_product_workspace(few)
    assert lib.kq8_product_workspace(few) % (64 * 1024 * 4) == 0 and lib.kq8_product_workspace(_shape(binding)) == 0
    assert lib.kq8_linear_workspace(_shape(binding, rows=0)) == 0 and lib.kq8_linear_workspace(_shape(binding, inner=131072)) == 0


def test_binding_refuses(binding):
    codes, scales = torch.zeros((4, 64), dtype=torch.int8), torch.zeros(4)
    with pytest.raises(ValueError):
        binding.kq8_rows(torch.zeros(4, 64))                # host memory
    with pytest.raises(ValueError):
        binding.kq8_product(codes, scales, codes, scales)
    with pytest.raises(ValueError):
        binding.kq8_linear(torch.zeros(4, 64), codes, scales)
