"""What the kernels' inline assembly tells the compiler (no GPU)."""
from __future__ import annotations

import glob
import os
import re

import pytest

from paper_2606_00024_amd import build


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(build.CSRC, "*"))), ids=os.path.basename)
def test_m0_is_the_compilers(path):
    """Loads into LDS take their place in m0 as an operand, and no statement writes m0
    itself: the compiler may keep values there."""
    with open(path) as f:
        statements = re.findall(r"__asm__[^;]*;", f.read())
    for s in statements:
        assert not re.search(r"\bs_\w+ m0,", s), s
        if "load_lds" in s:
            assert '"{m0}"(' in s, s
