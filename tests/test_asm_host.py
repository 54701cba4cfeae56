"""What the kernels' inline assembly tells the compiler (no GPU)."""
from __future__ import annotations

import glob
import os
import re

import pytest

from paper_2606_00024_amd import build


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(build.CSRC, "*"))), ids=os.path.basename)
def test_assembly_that_writes_m0_says_so(path):
    """A statement that sets m0 declares it: the compiler may keep values there."""
    with open(path) as f:
        statements = re.findall(r"__asm__[^;]*;", f.read())
    for s in statements:
        if re.search(r"\bs_\w+ m0,", s):
            assert re.search(r':[^:]*"m0"[^:]*\);$', s), s
