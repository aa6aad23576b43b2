"""Assembly statements in the kernels name what they write beside their operands."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1804_03243_amd", "csrc")


def statements():
    for f in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, f)).read()
        for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\);", text, re.S):
            yield f, m.group(1)


def test_written_registers_are_named():
    found = 0
    for f, s in statements():
        code, clobbers = s.split('"', 1)[1].rsplit('"v"', 1)[0], s.rsplit(":", 1)[-1]
        for reg in ("m0", "exec", "vcc", "scc"):
            if re.search(rf"\bs_mov\w*\s+{reg}\b", code):
                found += 1
                assert f'"{reg}"' in clobbers, (f, s)
    assert found
