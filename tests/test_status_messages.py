"""What a decode's status says (wd_status.h), on the host: each check that a kernel
makes of its own results has a text of its own, and all of them are WD_EDEVICE."""
import os
import subprocess

from paper_1804_03243_amd import wfstdec as wf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1804_03243_amd", "csrc")
SRC = r"""
#include <cstdio>
#include <initializer_list>
#include "wd_status.h"
int main() {
  for (int c = 0; c < 12; ++c)
    printf("%d|%s\n", wd::status_of(wd::internal_status(c)), wd::status_message(wd::internal_status(c)));
  for (int s : {WD_EINVAL, WD_ENOPATH, WD_ECAPACITY}) printf("%d|%s\n", wd::status_of(s), wd::status_message(s));
}
"""
CHECKS = ["kClusterWait", "kKeptCount", "kWarmPayload", "kGridFrame", "kSweepWait", "kLinkTarget", "kTraceback"]


def test_each_check_has_a_text(tmp_path):
    (tmp_path / "m.cpp").write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(tmp_path / "m"), str(tmp_path / "m.cpp")], check=True)
    lines = [l.split("|") for l in subprocess.run([str(tmp_path / "m")], capture_output=True, text=True, check=True).stdout.splitlines()]
    device, others = lines[:12], lines[12:]
    assert all(int(s) == wf.WD_EDEVICE and m.startswith("decode: a kernel's internal consistency check failed") for s, m in device)
    texts = [m for _, m in device[1:1 + len(CHECKS)]]
    assert len(set(texts + [device[0][1]])) == len(CHECKS) + 1
    assert all(m == device[0][1] for _, m in device[1 + len(CHECKS):])
    assert [int(s) for s, _ in others] == [wf.WD_EINVAL, wf.WD_ENOPATH, wf.WD_ECAPACITY]
    assert len({m for _, m in others}) == 3


def test_kernels_name_their_check():
    sources = "".join(open(os.path.join(CSRC, f)).read() for f in sorted(os.listdir(CSRC)) if f != "wd_status.h")
    assert "kStatusInternal" not in sources
    for check in CHECKS:
        assert check in sources, check
