"""Which arrays the projection may read eight elements at a time (wd_rows.h), on the
host: the last such load of an array must begin inside it."""
import ctypes
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r"""
#include "wd_rows.h"
extern "C" int shorter(long long rows, long long ld, long long n) { return wd::shorter_than_a_load(rows, ld, n); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "rows.cpp").write_text(SRC)
    out = str(d / "librows.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_1804_03243_amd", "csrc"),
                    "-o", out, str(d / "rows.cpp")], check=True)
    so = ctypes.CDLL(out)
    so.shorter.argtypes = [ctypes.c_longlong] * 3
    return so


def test_the_last_load_begins_inside_the_array(lib):
    for rows, n, gap in itertools.product(range(1, 12), range(1, 12), (0, 1, 2, 7, 100)):
        last = (rows - 1) * (n + gap) + n - 8
        assert bool(lib.shorter(rows, n + gap, n)) == (last < 0), (rows, n, gap)


def test_strides_near_the_largest(lib):
    assert not lib.shorter(2 ** 31 - 1, 2 ** 62, 1)
    assert lib.shorter(1, 2 ** 62, 7) and not lib.shorter(1, 2 ** 62, 8)
