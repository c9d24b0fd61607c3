"""What the kernel sources must not hold (CPU)."""
import glob
import os
import re

from tests.conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2608_15241_amd", "csrc")


def test_no_vector_arithmetic_in_inline_assembly():
    """The compiler puts the waits for the results of matrix products and exponentials before
    its own instructions only: arithmetic on vector registers is left to it."""
    found = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        for i, line in enumerate(open(path), 1):
            if re.search(r'asm\b[^"]*"\s*v_', line):
                found.append("%s:%d" % (os.path.basename(path), i))
    assert not found
