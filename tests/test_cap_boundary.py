"""Host-side checks of the attention and cache entry points that need no GPU: what is refused, before anything is launched."""
import ctypes
import os
import subprocess

import pytest

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
    values = dict(docs=1, q_rows=64, k_rows=64, heads=4, kv_heads=2, dim=64, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64,
                  scale=0.125, cap=50.0, window=0, causal=1)
    return binding.KcapShape(**{**values, **changes})


def _pages(binding, **changes):
    values = dict(page_size=16, page_count=8, most=4, table_row=4, k_page=2048, k_slot=128, k_head=64, v_page=2048, v_slot=128, v_head=64)
    return binding.KcapPages(**{**values, **changes})


def test_structures_have_the_headers_layout(binding, tmp_path):
    source, exe = tmp_path / "layout.c", tmp_path / "layout"
    fields = [(s, n) for s, c in (("kcap_shape_t", binding.KcapShape), ("kcap_pages_t", binding.KcapPages)) for n, _ in c._fields_]
    source.write_text('#include <stdio.h>\n#include "ktanh.h"\nint main(void) {\n' +
                      "".join(f'printf("%zu\\n", offsetof({s}, {n}));\n' for s, n in fields) +
                      'printf("%zu %zu\\n", sizeof(kcap_shape_t), sizeof(kcap_pages_t));\nreturn 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    mine = [getattr(c, n).offset for c in (binding.KcapShape, binding.KcapPages) for n, _ in c._fields_]
    assert [int(v) for v in out] == mine + [ctypes.sizeof(binding.KcapShape), ctypes.sizeof(binding.KcapPages)]


BAD_SHAPES = [(dict(dim=32), 4), (dict(dim=96), 4), (dict(heads=3), 4), (dict(heads=0), 4), (dict(kv_heads=0), 4), (dict(cap=0.0), 4), (dict(cap=-1.0), 4),
              (dict(cap=64.5), 4), (dict(cap=float("nan")), 4), (dict(scale=float("inf")), 4), (dict(scale=float("nan")), 4), (dict(q_rows=(1 << 30) + 1), 4),
              (dict(docs=1 << 40), 4), (dict(q_row=12), 2), (dict(v_head=4), 2), (dict(q_row=1 << 24), 4)]


def test_attention_refuses(binding):
    lib = binding.load_library()
    for name in ("kcap_attention", "kcap_attention64"):
        fn = getattr(lib, name)

        def call(shape, q=FAKE, k=FAKE, v=FAKE, q_at=FAKE, k_at=FAKE, o=FAKE, rest=NULL, lse=NULL, lut=None):
            return fn(shape, q, k, v, q_at, k_at, o, rest, lse, lut, NULL)
        assert call(None) == 1
        assert call(_shape(binding, q_rows=0), q=NULL, o=NULL) == 0 and call(_shape(binding, docs=0)) == 0
        for missing in ("q", "k", "v", "q_at", "k_at", "o"):
            assert call(_shape(binding), **{missing: NULL}) == 1, missing
        for bad, status in BAD_SHAPES:
            assert call(_shape(binding, **bad)) == status, bad
        assert call(_shape(binding, k_rows=(1 << 30) + 1)) == 4
        for off in ("q", "k", "v"):
            assert call(_shape(binding), **{off: ctypes.c_void_p(0x1008)}) == 2
        for off in ("o", "rest"):
            assert call(_shape(binding), **{off: ctypes.c_void_p(0x1004)}) == 2
        assert call(_shape(binding), lse=ctypes.c_void_p(0x1002)) == 2 and call(_shape(binding), q_at=ctypes.c_void_p(0x1002)) == 2
        assert call(_shape(binding, q_rows=1 << 30, heads=64, kv_heads=64)) == 4       # more blocks than a launch holds
    table = binding.ktanh_default_lut()
    table.r[5] = 9
    assert lib.kcap_attention(_shape(binding), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, NULL, NULL, table, NULL) == 3
    table = binding.ktanh_default_lut()
    table.E[31], table.b[31] = 127, 0               # valid by itself, but K would be above 1 on [1.875, 2)
    assert binding.ktanh_lut_validate(table) == 0
    assert lib.kcap_attention(_shape(binding), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, NULL, NULL, table, NULL) == 3


def test_gradients_refuse(binding):
    lib = binding.load_library()
    for name in ("kcap_attention_backward", "kcap_attention64_backward"):
        fn = getattr(lib, name)

        def call(shape, do_row=256, do_head=64, lut=None, **changes):
            names = ("d_o", "q", "k", "v", "o", "rest", "lse", "q_at", "k_at", "dq", "dk", "dv", "work")
            p = {n: FAKE for n in names} | {"rest": NULL} | changes
            return fn(shape, p["d_o"], do_row, do_head, *(p[n] for n in names[1:]), lut, NULL)
        assert call(None) == 1
        assert call(_shape(binding, docs=0)) == 0 and call(_shape(binding, q_rows=0, k_rows=0)) == 0
        for missing in ("d_o", "q", "k", "v", "o", "lse", "q_at", "k_at", "dq", "dk", "dv", "work"):
            assert call(_shape(binding), **{missing: NULL}) == 1, missing
        for bad, status in BAD_SHAPES:
            assert call(_shape(binding, **bad)) == status, bad
        assert call(_shape(binding), do_row=12) == 2 and call(_shape(binding), do_head=1 << 24) == 4
        for off in ("d_o", "o", "rest", "dq", "dk", "dv", "work"):
            assert call(_shape(binding), **{off: ctypes.c_void_p(0x1008)}) == 2, off
    assert lib.kcap_attention_backward_workspace(_shape(binding)) >= 64 * 4 * 4       # delta
    size = lib.kcap_attention_backward_workspace(_shape(binding, q_rows=8192, k_rows=8192))
    assert size >= 8192 * 4 * 4 + 2 * 2 * 8192 * 2 * 64 * 4       # delta, and a part for each of two shared heads
    assert lib.kcap_attention_backward_workspace(None) == 0


BAD_PAGES = [(dict(page_size=0), 4), (dict(page_size=12), 4), (dict(page_size=1 << 21), 4), (dict(page_count=0), 4), (dict(most=0), 4),
             (dict(most=1 << 30), 4), (dict(k_page=12), 2), (dict(v_head=4), 2), (dict(k_page=1 << 31), 4)]


def test_paged_attention_refuses(binding):
    lib = binding.load_library()
    one = dict(docs=64, k_rows=0)
    for name in ("kcap_attention_paged", "kcap_attention64_paged"):
        fn = getattr(lib, name)

        def call(shape, cache, q_at=NULL, lut=None, **changes):
            p = {n: FAKE for n in ("q", "k", "v", "pages", "lengths", "o", "work")} | changes
            return fn(shape, cache, p["q"], p["k"], p["v"], p["pages"], p["lengths"], q_at, p["o"], p["work"], lut, NULL)
        good = _pages(binding)
        assert call(None, good) == 1 and call(_shape(binding, **one), None) == 1
        assert call(_shape(binding, docs=0), good) == 0 and call(_shape(binding, q_rows=0), good) == 0
        for missing in ("q", "k", "v", "pages", "lengths", "o", "work"):
            assert call(_shape(binding, **one), good, **{missing: NULL}) == 1, missing
        for bad, status in BAD_SHAPES:
            if "k_rows" not in bad and "docs" not in bad and "q_rows" not in bad and "v_head" not in bad:
                assert call(_shape(binding, **{**one, **bad}), good) == status, bad
        for bad, status in BAD_PAGES:
            assert call(_shape(binding, **one), _pages(binding, **bad)) == status, bad
        for off in ("q", "k", "v", "work"):
            assert call(_shape(binding, **one), good, **{off: ctypes.c_void_p(0x1008)}) == 2, off
        assert call(_shape(binding, docs=63), good) == 4      # one query each, but not as many queries as sequences
        assert call(_shape(binding, **one), good, q_at=ctypes.c_void_p(0x1002)) == 2
        assert call(_shape(binding, docs=1 << 20, q_rows=1 << 20), _pages(binding, most=1 << 26)) == 4      # more tiles than 32 bits number
    assert lib.kcap_attention_paged_workspace(_shape(binding, **one), _pages(binding), 1) > 0
    assert lib.kcap_attention_paged_workspace(None, _pages(binding), 1) == 0
    few = _shape(binding, docs=1, q_rows=3)
    assert lib.kcap_attention_paged_workspace(few, _pages(binding, most=4096), 0) > 0       # one piece of a long text: keys are shared out
    assert lib.kcap_attention_paged_workspace(few, _pages(binding), 0) == 0


def test_append_refuses(binding):
    lib = binding.load_library()

    def call(shape, cache, q_at=FAKE, positions=32, angles=32, **changes):
        p = {n: FAKE for n in ("q", "k", "v", "out", "kc", "vc", "pages", "lengths", "cos", "sin")} | changes
        return lib.kcap_append(shape, cache, p["q"], p["k"], p["v"], p["out"], p["kc"], p["vc"], p["pages"], p["lengths"], q_at, p["cos"], p["sin"],
                               positions, angles, 0, NULL)
    good = _pages(binding)
    assert call(None, good) == 1 and call(_shape(binding), None) == 1
    assert call(_shape(binding, q_rows=0), good) == 0 and call(_shape(binding, docs=0), good) == 0
    for missing in ("q", "k", "v", "out", "kc", "vc", "pages", "lengths", "cos", "sin"):
        assert call(_shape(binding), good, **{missing: NULL}) == 1, missing
    for bad, status in BAD_PAGES:
        assert call(_shape(binding), _pages(binding, **bad)) == status, bad
    for off in ("q", "k", "v", "out", "kc", "vc", "cos", "sin"):
        assert call(_shape(binding), good, **{off: ctypes.c_void_p(0x1008)}) == 2, off
    assert call(_shape(binding), good, angles=12) == 4 and call(_shape(binding), good, angles=40) == 4 and call(_shape(binding), good, angles=0) == 4
    assert call(_shape(binding), good, positions=0) == 4 and call(_shape(binding), good, q_at=NULL) == 4
    assert call(_shape(binding, dim=48), good) == 4 and call(_shape(binding, q_row=20), good) == 2


@pytest.mark.parametrize("scale,cap", [(1.0, 1e-40), (1e300, 50.0), (-1e30, 1e-10), (1e39, 64.0)])
def test_a_scale_over_cap_beyond_float32_is_refused(binding, scale, cap):
    """An infinite factor gives NaN for a score of zero, and an infinite argument for one that saturates."""
    lib = binding.load_library()
    options = dict(scale=scale, cap=cap)
    some = [FAKE] * 6
    assert lib.kcap_attention(_shape(binding, **options), *some, NULL, NULL, None, NULL) == 4
    assert lib.kcap_attention64(_shape(binding, **options), *some, NULL, NULL, None, NULL) == 4
    assert lib.kcap_attention_backward(_shape(binding, **options), FAKE, 256, 64, *[FAKE] * 4, NULL, *[FAKE] * 7, None, NULL) == 4
    for q_at in (NULL, FAKE):
        assert lib.kcap_attention_paged(_shape(binding, docs=64, k_rows=0, **options), _pages(binding), *[FAKE] * 5, q_at, FAKE, FAKE, None, NULL) == 4


def test_lines_of_k_under_sanitizers(tmp_path):
    """The packing of K-TanH's tables as lines, with ASan and UBSan: on every interval the line is Algorithm 1's value."""
    csrc = os.path.join(ROOT, "paper_1909_07729_amd", "csrc")
    exe = tmp_path / "cap_lines"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-I",
                    os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "host_c", "cap_lines.cpp"),
                    os.path.join(csrc, "ktanh_lut.cpp"), os.path.join(csrc, "ktanh_fit.cpp"), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0 and "lines agree" in res.stdout, res.stdout + res.stderr
