"""Inline assembly in the kernels' sources: registers that it writes by name are known to the compiler (no GPU)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_26253_amd", "csrc")


def statements(text):
    """The inline assembly of a source: everything between the parentheses of asm and asm volatile."""
    for m in re.finditer(r"\basm\s+(?:volatile\s*)?\(|\basm\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text[m.end():at - 1]


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h*"))), ids=os.path.basename)
def test_what_assembly_writes_by_name_is_a_clobber(path):
    """A register that an instruction names as its destination is on the statement's list (m0, reserved, comes in as an operand
    instead: "{m0}")."""
    with open(path) as f:
        text = f.read()
    for s in statements(text):
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', s.split(":")[0])).replace("\\n", "\n").replace("\\t", " ")
        for line in code.split("\n"):
            m = re.match(r"\s*([sv]_\w+)\s+(m0|vcc|exec|s\d+|v\d+|s\[\d+:\d+\]|v\[\d+:\d+\])\b", line)
            if m and not m.group(1).startswith("s_waitcnt"):
                assert f'"{m.group(2)}"' in s.rsplit(":", 1)[-1], line
