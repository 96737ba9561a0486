"""Inline assembly in the kernels' sources names what it changes: a special register that it writes stands
among its clobbers, so that the compiler keeps nothing there."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2007_06563_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.h*")))


def statements(text):
    """The asm statements of a source: what stands between their outer parentheses."""
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        yield text[m.end():i - 1]


def written(statement):
    """Special registers that instructions of a statement name as their target."""
    code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', statement.split("\n:")[0]))
    return {w for line in re.split(r"\\n|;", code)
            for w in re.findall(r"^\s*(?:\\t)*[sv]_\w+\s+(m0|vcc|exec)\b", line.replace("\\t", " "))}


def test_the_search_itself():
    found = list(statements('asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0" : : "s"(f(x)) : "memory", "m0");'))
    assert len(found) == 1 and written(found[0]) == {"m0"}
    assert written('"s_waitcnt vmcnt(0)" ::: "memory"') == set()


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_written_registers_are_clobbers(path):
    for st in statements(open(path).read()):
        for reg in written(st):
            assert f'"{reg}"' in st, (path, reg, st)
