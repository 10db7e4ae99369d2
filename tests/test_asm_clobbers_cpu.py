"""Assembly that sets m0 for its own use names it as clobbered: the compiler may
hold a value of its own there."""
import glob
import os
import re

from paper_2007_00072_amd import build


def test_m0_is_named():
    seen = 0
    for path in glob.glob(os.path.join(build.CSRC, "*.h*")):
        for asm in re.findall(r"asm volatile\((.*?)\);", open(path).read(), flags=re.S):
            if "s_mov_b32 m0" in asm:
                seen += 1
                assert '"m0"' in asm, (os.path.basename(path), asm)
    assert seen >= 3
