"""Statements of instructions written in asm leave m0 as they found it (CPU): the
compiler keeps values of its own there, and a clobber of a register that is not its to
allocate does not bind it."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_1903_01814_amd", "csrc")


def statements(text):
    """The instructions of every asm statement."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r'\basm\b(?:\s+volatile)?\s*\(((?:\s*"(?:[^"\\]|\\.)*")+)', text):
        lines = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', m.group(1)))
        yield [i.strip() for i in re.split(r"\\n|\\t|;", lines) if i.strip()]


def puts_back(lines):
    """m0 is not changed, or is saved first and restored last."""
    if not any(re.match(r"s_\w+\s+m0\b", i) for i in lines):
        return True
    first = re.fullmatch(r"s_mov_b32 (%\d+), m0", lines[0])
    return bool(first) and lines[-1] == "s_mov_b32 m0, %s" % first.group(1)


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h*"))),
                         ids=os.path.basename)
def test_m0_is_put_back(path):
    with open(path) as f:
        for lines in statements(f.read()):
            assert puts_back(lines), lines


@pytest.mark.parametrize("text,good", [
    (r'asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\t" "x %2\n\ts_mov_b32 m0, %0" : "=&s"(w)',
     True),
    (r'asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tx %1, %2" ::"s"(to), "v"(a) : "m0");', False),
    (r'asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_mov_b32 m0, %1" : "=&s"(w)', False),
    (r'asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");', True)])
def test_the_scan_sees_it(text, good):
    lines, = statements(text)
    assert len(lines) >= 2 and puts_back(lines) == good
