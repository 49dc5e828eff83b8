"""Barriers written in inline asm (no GPU).  The compiler's own barrier waits for a wave's LDS accesses; one in asm does so only if it says so.  A wave that arrives with reads of
LDS under way lets the others overwrite what it reads, so each of them waits for lgkmcnt(0) in the same statement."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_10700_amd", "csrc")


def test_barriers_in_asm_wait_for_lds():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if not path.endswith((".h", ".hip", ".cpp", ".inc")):
            continue
        for text in re.findall(r'asm\s+volatile\s*\(\s*((?:"[^"]*"\s*)+)', open(path).read()):
            if "s_barrier" in text:
                found += 1
                assert re.search(r"s_waitcnt[^;]*lgkmcnt\(0\).*s_barrier", text), (os.path.basename(path), text)
    assert found >= 4
