"""How products in 8-bit integers are cut into blocks: a program of the host's own code prints the plans."""
import os
import subprocess

import pytest

from conftest import ROOT
from test_gpu_q8 import TILES

KINDS = [(256, 256), (192, 256), (128, 128), (128, 64), (64, 64), (128, 32), (16, 16)]     # channels, rows


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "q8_plans")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_1909_07729_amd", "csrc"), os.path.join(ROOT, "tests", "host_c", "q8_plans.cpp"), "-o", exe], check=True)

    def of(shapes):
        lines = subprocess.run([exe], input="".join(f"{r} {i} {o}\n" for r, i, o in shapes), text=True, capture_output=True, check=True).stdout.split("\n")
        return [tuple(map(int, line.split())) for line in lines if line]
    return of


def test_the_tests_of_tiles_reach_every_kind(plans):
    got = plans(TILES)
    assert [(over, across, parts) for _, over, across, parts, _ in got] == [
        (256, 256, 1), (192, 256, 1), (128, 128, 1), (128, 128, 1), (128, 64, 1), (64, 64, 1), (128, 32, 1), (128, 32, 1), (128, 64, 4), (64, 64, 8), (64, 64, 8)]
    blocks = [-(-o // over) * -(-r // across) * parts for (r, _, o), (_, over, across, parts, _) in zip(TILES, got)]
    assert blocks[2] > 256 >= blocks[3]        # tiles of 128 by 128 with two places and with three


def test_plans_over_the_range(plans):
    sizes = [1, 2, 15, 16, 17, 64, 100, 511, 512, 1000, 4096, 10000, 1 << 20, 1 << 30]
    shapes = [(r, i, o) for r in sizes for o in sizes for i in (0, 1, 127, 128, 1000, 4096, 16384, 131071)]
    for (rows, inner, outer), (kind, over, across, parts, sums) in zip(shapes, plans(shapes), strict=True):
        assert KINDS[kind] == (over, across)
        assert parts == 1 or (parts in (2, 4, 8) and inner // 128 >= 4 * parts and kind in (2, 3, 4, 5))
        assert sums == (parts * rows * outer * 4 if parts > 1 else 0)
        if parts > 1:       # sums of parts are for few results: what is written and read again stays a small part of the call
            assert sums <= 1 << 28


def test_one_row_and_none(plans):
    assert plans([(0, 4096, 4096), (4096, 4096, 0), (1, 0, 1)])[0][4] == 0
    assert plans([(1, 4096, 4096)])[0][0] == 6
