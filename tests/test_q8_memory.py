"""Calls on 8-bit integers whose outputs share memory with what they read: refused on the host, before anything is launched."""
import ctypes
import os
import random
import subprocess

import pytest

from conftest import ROOT
from test_q8_boundary import NULL, _shape, binding  # noqa: F401


def _bytes(at, rows, size, step):
    return {at + r * step + i for r in range(rows) for i in range(size)}


def test_what_is_apart(tmp_path):
    """Against the bytes themselves: never apart where they meet, and always apart where spans do not cross or rows of one stride lie beside each other."""
    exe = str(tmp_path / "q8_memory")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_1909_07729_amd", "csrc"), os.path.join(ROOT, "tests", "host_c", "q8_memory.cpp"), "-o", exe], check=True)
    rng = random.Random(1)
    cases = []
    for _ in range(60000):
        step = rng.randint(1, 20)
        pair = []
        for _ in range(2):
            rows = rng.choice([1, 1, 2, 3, 5])
            pair.append((rng.randint(1, 90), rows, rng.randint(0, 12), 0 if rows == 1 else rng.choice([step, step, rng.randint(1, 20)])))
        cases.append(pair)
    lines = "".join(" ".join(map(str, a + b)) + "\n" for a, b in cases)
    got = [line == "1" for line in subprocess.run([exe], input=lines, text=True, capture_output=True, check=True).stdout.split()]
    counts = [0, 0, 0]
    for (a, b), answer in zip(cases, got, strict=True):
        x, y = _bytes(*a), _bytes(*b)
        crossing = x and y and min(x) <= max(y) and min(y) <= max(x)
        if x & y:
            assert not answer, (a, b)
            counts[0] += 1
        elif not crossing:
            assert answer, (a, b)
            counts[1] += 1
        elif a[1] > 1 and b[1] > 1 and a[3] == b[3]:
            # beside each other: no row of either would meet one of the other's however many they were
            endless = _bytes(a[0] % a[3] + a[3], 1, a[2], 0) & set().union(*(_bytes(b[0] % a[3] + k * a[3], 1, b[2], 0) for k in range(4)))
            assert answer == (not endless and a[2] <= a[3] and b[2] <= a[3]), (a, b)
            counts[2] += 1
    assert min(counts) > 500
    far = [(1 << 47, 1 << 30, 1 << 30, 1 << 42), (1, 1, 8, 0), (1 << 46, 1, 1 << 40, 0)]        # spans past 64 bits
    lines = "".join(" ".join(map(str, far[i] + far[j])) + "\n" for i, j in ((0, 1), (0, 2), (1, 2), (0, 0)))
    assert subprocess.run([exe], input=lines, text=True, capture_output=True, check=True).stdout.split() == ["1", "1", "1", "0"]


X, W, S, T, B, OUT, WORK = (ctypes.c_void_p(i << 24) for i in range(1, 8))      # never dereferenced: refused on the host


def _near(pointer, by=0):
    return ctypes.c_void_p(pointer.value + by)


def test_calls_refuse(binding):
    lib = binding.load_library()
    for rows, inner, outer in ((8, 64, 32), (300, 512, 512)):       # one launch, and two
        shape = _shape(binding, rows=rows, inner=inner, outer=outer, x_row=inner, w_row=inner, out_row=outer)
        for name in ("kq8_linear", "kq8_linear64"):
            for out in (X, _near(X, 2 * rows * inner - 2), W, T, B, _near(T, 4 * outer - 4), _near(X, -2)):
                assert getattr(lib, name)(shape, X, W, T, B, out, WORK, None, NULL) == 4, (name, out)
        for out in (X, _near(X, rows * inner - 2), W, S, T, B):
            assert lib.kq8_product(shape, X, S, W, T, B, out, WORK, NULL) == 4, out
        for name in ("kq8_rows", "kq8_rows64"):
            for codes, scales in ((X, S), (_near(X, 8), S), (W, X), (W, _near(W, 4)), (W, _near(W, rows * inner - 4))):
                assert getattr(lib, name)(shape, X, codes, inner, scales, None, NULL) == 4, (name, codes, scales)
    # rows of two strides that cross, and of one stride that meet
    wide = _shape(binding, x_row=256, out_row=200)
    assert lib.kq8_linear(wide, X, W, T, B, _near(X, 128), WORK, None, NULL) == 4
    wide = _shape(binding, x_row=256, out_row=256)
    assert lib.kq8_linear(wide, X, W, T, B, _near(X, 126), WORK, None, NULL) == 4
    assert lib.kq8_linear(wide, X, W, T, B, _near(X, 512 * 3 + 512 - 62), WORK, None, NULL) == 4
