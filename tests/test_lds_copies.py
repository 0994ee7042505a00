"""Copies from global memory to LDS take their LDS address from m0, which needs
a wait state after it has been written (the compiler sees to it in its own code,
not inside inline assembly): each statement that does both has it."""

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14530_amd", "csrc")


def statements():
    """(file, instructions) of the inline assembly that writes m0"""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        for m in re.finditer(r"asm\s+volatile\s*\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", open(path).read()):
            text = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))
            lines = [s.strip() for s in re.split(r"\\n|;|\\t", text) if s.strip()]
            if any(re.match(r"s_\w+ m0\b", s) for s in lines):
                yield os.path.basename(path), lines


def is_copy(s):
    return re.match(r"(global_load_lds|scratch_load_lds)", s) or (s.startswith("buffer_load") and s.endswith("lds"))


def test_the_statements_are_found():
    names = [n for n, lines in statements() for s in lines if is_copy(s)]
    assert names.count("xhc_device.h") == 2 and names.count("xhc_ffn.h") == 1


@pytest.mark.parametrize("name,lines", list(statements()))
def test_m0_is_waited_for(name, lines):
    written = None
    for i, s in enumerate(lines):
        if re.match(r"s_\w+ m0\b", s):
            written = i
        if is_copy(s) and written is not None:
            between = lines[written + 1:i]
            assert between and between[0].startswith("s_nop"), (name, lines)
