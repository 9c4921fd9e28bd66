"""Inline assembly that gives a memory instruction a scalar base waits for it: the
register may have been written by a vector instruction just before (readfirstlane),
which takes five wait states, and the compiler does not look into the statement."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_24593_amd", "csrc")


def waits(statement):
    """Wait states before the first memory instruction of an asm statement."""
    before = re.split(r"(?:global|buffer|flat)_", statement)[0]
    return sum(int(n) + 1 for n in re.findall(r"s_nop (\d+)", before))


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h*"))), ids=os.path.basename)
def test_scalar_bases_are_waited_for(path):
    with open(path) as f:
        text = f.read()
    for statement in re.findall(r"asm volatile\((.*?)\);", text, re.S):
        if re.search(r"(?:global|buffer|flat)_", statement) and re.search(r'"s"\(', statement):
            assert waits(statement) >= 5, (os.path.basename(path), statement)


def test_what_is_found():
    assert waits('"s_nop 0\\n\\tglobal_load_lds_dwordx4 %1, %2"') == 1
    assert waits('"s_nop 4\\n\\tglobal_load_lds_dwordx4 %1, %2"') == 5
