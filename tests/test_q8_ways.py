"""Which kernel a product in 8-bit integers takes, and the launches that it is cut into: a program of the host's own code prints them."""
import os
import subprocess

import pytest

from conftest import ROOT

TILES, SHARED16, SHARED64 = range(3)


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("ways") / "q8_ways")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_1909_07729_amd", "csrc"), os.path.join(ROOT, "tests", "host_c", "q8_ways.cpp"), "-o", exe], check=True)

    def of(calls):
        lines = subprocess.run([exe], input="".join(" ".join(map(str, c)) + "\n" for c in calls), text=True, capture_output=True, check=True).stdout.split("\n")
        return [tuple(map(int, line.split())) for line in lines if line]
    return of


def test_every_launch_fits_its_grid(ways):
    """Fewer than 2^32 lanes along the blocks' first dimension and at most 65535 blocks along the second; one launch wherever that is enough."""
    sizes = [1, 2, 16, 17, 33, 64, 1000, 4096, 65535 * 16, 65535 * 16 + 1, 65535 * 64, 65535 * 64 + 1, 1 << 24, 1 << 27, (1 << 27) + 1, (1 << 30) - 1, 1 << 30]
    calls = [(r, i, o, a, s, s) for r in sizes for o in sizes for i in (0, 1, 128, 1000, 131071) for a in (0, 1) for s in (131072, 1 << 23)]
    split = set()
    for (rows, _, outer, aligned, step, _), (way, over, across, parts, piece_rows, piece_outer) in zip(calls, ways(calls), strict=True):
        assert way != TILES or (aligned and step < 1 << 23)
        over, across, lanes = (over, across, 256) if way == TILES else (16, 16, 512) if way == SHARED16 else (64, 64, 256)

        def fits(r, o):
            x, y = -(-o // over), -(-r // across)
            return x * y * parts * lanes < 1 << 32 if way == TILES else x * lanes < 1 << 32 and y <= 65535
        assert 1 <= piece_rows <= rows and 1 <= piece_outer <= outer and fits(piece_rows, piece_outer)
        assert (piece_rows == rows or piece_rows % across == 0) and (piece_outer == outer or piece_outer % over == 0)
        assert (piece_rows == rows and piece_outer == outer) == fits(rows, outer)
        if not fits(rows, outer):
            split.add((way, piece_rows < rows, piece_outer < outer))
    assert {(SHARED16, False, True), (SHARED64, True, False), (TILES, True, False)} <= split


def test_the_tests_of_many_rows_and_channels_take_several_launches(ways):
    from test_gpu_q8_many import PRODUCTS
    for (rows, inner, outer, aligned), (way, *_, piece_rows, piece_outer) in zip(PRODUCTS, ways([(*p, 17 - p[3], 17 - p[3]) for p in PRODUCTS]), strict=True):
        assert (way == TILES) == bool(aligned) and (piece_rows < rows or piece_outer < outer)


def test_the_tests_off_the_grid_reach_the_blocks_of_64(ways):
    from test_gpu_q8_off_grid import FAR, OFF_GRID

    def on_grid(inner, apart, start):
        return start % 16 == 0 and (inner + apart) % 16 == 0
    calls = [(r, i, o, int(on_grid(i, xa, xs) and on_grid(i, wa, ws)), i + xa, i + wa) for r, i, o, xa, xs, wa, ws in OFF_GRID]
    assert not any(c[3] for c in calls)
    far = [(r, i, o, 1, x, w) for r, i, o, x, w in FAR]
    assert all(x % 16 == w % 16 == 0 for *_, x, w in FAR)
    assert all(way == SHARED64 for way, *_ in ways(calls + far))
    assert ways([(600, 1001, 1000, 0, 1008, 1001)])[0][0] == SHARED64
