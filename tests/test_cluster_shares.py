"""Which frames of a cluster of workgroups end with a barrier (wd_spin.h), on the host:
all whose shares of the touched states are more than a workgroup holds."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r"""
#include "wd_spin.h"
extern "C" int held(unsigned n, unsigned N, unsigned each) { return wd::shares_held(n, N, each); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("shares")
    (d / "shares.cpp").write_text(SRC)
    out = str(d / "libshares.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_1804_03243_amd", "csrc"),
                    "-o", out, str(d / "shares.cpp")], check=True)
    return ctypes.CDLL(out)


def largest_share(n, N):
    return max(n * (w + 1) // N - n * w // N for w in range(N))


@pytest.mark.parametrize("N", [1, 2, 7, 31, 32])
def test_a_list_read_again_is_found(lib, N):
    each = 3072
    for n in [0, 1, each - 1, each, each + 1, 1_000_000, 2 ** 32 - 1] + [N * each + k for k in range(-3, 4)]:
        assert bool(lib.held(n, N, each)) == (largest_share(n, N) <= each), n
