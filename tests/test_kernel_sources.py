"""What the kernels' inline assembly has to tell the compiler, read from the sources (no GPU)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2011_13824_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.h*")))


def statements(text):
    """(instructions, constraints) of every asm statement."""
    for m in re.finditer(r"asm volatile\((.*?)\);", text, re.S):
        code = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', m.group(1)).group(1)
        yield code, m.group(1)[len(code):]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_assembly_names_what_it_writes(path):
    for code, constraints in statements(open(path).read()):
        if re.search(r"\bs_mov_b32 m0\b", code):
            assert '"m0"' in constraints, code
        if re.search(r"\blds\b|s_barrier|s_waitcnt", code):
            assert '"memory"' in constraints, code


def test_statements_are_found():
    found = [c for p in SOURCES for c, _ in statements(open(p).read())]
    assert sum("m0" in c for c in found) >= 2 and any("s_barrier" in c for c in found)
