"""What the compiler does not see of the inline assembly in the kernels of the 4-bit microscaled operators, without a GPU."""
import glob
import os
import re

import pytest

from test_inline_asm import CSRC, _asm_texts

SOURCES = sorted(glob.glob(os.path.join(CSRC, "mx4*.hip")))


def _statements(path):
    with open(path) as f:
        return _asm_texts(f.read())


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_a_barrier_waits_for_the_lds_reads_before_it(path):
    """LDS that waves read before a barrier is written by others behind it.  The compiler waits for a read where its result
    is used, which may be behind a barrier that it cannot see, so the statement with the barrier has to."""
    for asm in _statements(path):
        before, barrier, _ = asm.partition("s_barrier")
        assert not barrier or "lgkmcnt(0)" in before, asm


def test_the_barriers_are_found():
    assert sum("s_barrier" in asm for path in SOURCES for asm in _statements(path)) >= 3


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_m0_is_an_operand_of_what_reads_it(path):
    """A load to LDS takes its address from m0.  The compiler has to know of a value there, or it may have one of its
    own in the register across the statement."""
    with open(path) as f:
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    for statement in re.findall(r"\basm\b[^;]*;", text, flags=re.S):
        assert not re.search(r"\bs_\w+ m0\b", statement), statement
        assert "load_lds" not in statement or '"{m0}"' in statement, statement
