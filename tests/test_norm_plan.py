"""The host's choice of the non-temporal hint for the norm (csrc/plan.h), checked without a GPU through a small C++ shim."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "plan.h"
extern "C" int streams(int bytes, int rows, int cols, int tensors, long s0, long s1, long s2) { return spes::plan::norm_streams(bytes, rows, cols, tensors, s0, s1, s2); }
"""


@pytest.fixture(scope="module")
def streams(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared",
                    "-fPIC", "-I", os.path.join(ROOT, "paper_2602_11543_amd", "csrc"), str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    fn = ctypes.CDLL(str(d / "shim.so")).streams
    fn.argtypes = [ctypes.c_int] * 4 + [ctypes.c_long] * 3
    return lambda bytes, rows, cols, tensors, *s: bool(fn(bytes, rows, cols, tensors, *(s or (cols, cols, cols))))


@pytest.mark.parametrize("rows,cols", [(524288, 4096), (1048576, 2048), (131072, 16384), (1 << 30, 64), (2 ** 31 - 1, 16384)])
def test_largest_streams(streams, rows, cols):
    """Beyond 2^31 elements."""
    for bytes in (2, 4):
        for tensors in (2, 3, 4):
            assert streams(bytes, rows, cols, tensors)


def test_where_the_cache_ends(streams):
    assert streams(2, 32768, 4096, 4) and not streams(2, 32768, 1024, 4) and streams(2, 32769, 1024, 4)
    assert not streams(4, 4096, 768, 4) and not streams(2, 0, 4096, 4)


def test_rows_that_end_inside_a_line(streams):
    assert not streams(2, 65536, 4104, 4) and not streams(2, 65536, 4096, 4, 4104, 4096, 4096) and not streams(4, 65536, 4096, 4, 4096, 4096, 4100)
    assert streams(4, 65536, 4096, 4, 4128, 4096, 0)
