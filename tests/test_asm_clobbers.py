"""Inline assembly that writes a special register by name lists it as clobbered."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_24593_amd", "csrc")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h*"))), ids=os.path.basename)
def test_special_registers_are_clobbered(path):
    with open(path) as f:
        text = f.read()
    for statement in re.findall(r"asm volatile\((.*?)\);", text, re.S):
        for reg in re.findall(r"s_mov_b(?:32|64) (m0|vcc|exec)\b", statement):
            assert re.search(rf'"{reg}"', statement), (os.path.basename(path), statement)
