"""The host's choice of tiles for the orthogonalisation's products (csrc/plan.h), checked without a GPU through a small C++ shim."""
import ctypes
import os
import subprocess

import pytest

from test_gpu_orthogonalize import PARTS, SIDES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "plan.h"
extern "C" int square_tile(int rows, int cols, int n, int symmetric) { return spes::plan::square_tile(rows, cols, n, symmetric != 0); }
extern "C" int square_cut(int side, int count) { return (int)spes::plan::square_cut(side, count); }
extern "C" int gram_parts(int lo, int hi, int n, int pairs) { return spes::plan::gram_parts(lo, hi, n, pairs != 0); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2602_11543_amd", "csrc"),
                    str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    return ctypes.CDLL(str(d / "shim.so"))


@pytest.fixture(scope="module")
def square_tile(lib):
    return lib.square_tile


@pytest.mark.parametrize("n,rows,cols,side", SIDES)
def test_device_tests_reach_every_tile(square_tile, n, rows, cols, side):
    lo, hi = (-(-v // 64) * 64 for v in sorted((rows, cols)))
    assert square_tile(lo, hi, n, 0) == side and square_tile(lo, lo, n, 1) == side


@pytest.mark.parametrize("rows,cols,n,symmetric,want", [
    (3584, 4864, 8, 0, 256), (3584, 3584, 8, 1, 256), (1024, 2048, 16, 0, 256), (1024, 1024, 16, 1, 256),      # rounds of full tiles
    (1280, 1536, 1, 0, 128), (2048, 2048, 1, 0, 128),                                                         # one block per CU of half as wide ones
    (256, 512, 4, 0, 64), (256, 256, 4, 1, 64), (64, 64, 1, 1, 64), (1280, 1280, 1, 1, 64), (64, 16384, 1, 0, 64)])
def test_sides(square_tile, rows, cols, n, symmetric, want):
    assert square_tile(rows, cols, n, symmetric) == want


def test_never_more_than_a_round_dearer_than_full_tiles(square_tile):
    """Full tiles of one round are left only for tiles that are one round as well, or nearly."""
    for n in (1, 2, 5, 16, 60):
        for lo in range(64, 2049, 64):
            for hi in (lo, 2 * lo):
                full = -(-lo // 256) * -(-hi // 256) * n
                side = square_tile(lo, hi, n, 0)
                small = -(-lo // side) * -(-hi // side) * n
                assert side == 256 or small <= 1024 * -(-full // 256)


def test_halves(lib):
    """Of 256-wide tiles a last round of 256, of others of 512, that has at most one tile for every second CU."""
    for side, count, want in [(256, 840, 72), (256, 896, 128), (256, 897, 0), (256, 512, 0), (128, 120, 120), (128, 129, 0), (128, 512 + 64, 64),
                              (128, 512, 0), (64, 100, 100), (64, 150, 0)]:
        assert lib.square_cut(side, count) == want, (side, count)


def test_device_tests_reach_halves(lib, square_tile):
    reached = set()
    for n, rows, cols, side in SIDES + [(1, 1100, 1300, 128)]:
        lo, hi = (-(-v // 64) * 64 for v in sorted((rows, cols)))
        mt, nt = -(-lo // side), -(-hi // side)
        for symmetric, count in ((0, mt * nt * n), (1, mt * (mt + 1) // 2 * n)):
            cut = lib.square_cut(side, count)
            reached |= {(side, symmetric, kind) for kind, tiles in (("whole", count - cut), ("halves", cut)) if tiles}
    assert reached == {(side, symmetric, kind) for side in (256, 128, 64) for symmetric in (0, 1) for kind in ("whole", "halves")}


@pytest.mark.parametrize("n,rows,cols,parts", PARTS + [(1, 64, 1344, 1), (40, 64, 4864, 1), (1, 512, 4864, 1), (32, 64, 4864, 4)])
def test_parts(lib, n, rows, cols, parts):
    """Few tiles with a long contraction; every part has K-tiles, and halves of all the tiles at once have a CU each."""
    lo, hi = (-(-v // 64) * 64 for v in sorted((rows, cols)))
    assert lib.gram_parts(lo, hi, n, 1) == parts and lib.gram_parts(lo, hi, n, 0) == (parts if hi // 64 >= 44 else 1)
    each = -(-(hi // 64) // parts)
    assert (parts - 1) * each < hi // 64 and (parts == 1 or parts * n * (lo // 64) * (lo // 64 + 1) <= 256)
