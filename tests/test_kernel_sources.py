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


def kernels():
    """(name, metadata) of the kernels in the built library: the notes of the code objects that it holds."""
    msgpack = pytest.importorskip("msgpack")
    import struct

    import paper_2607_26253_amd as sara
    with open(sara.LIB_PATH, "rb") as f:
        data = f.read()
    at = data.find(b"\x7fELF", 1)
    while at > 0:
        if struct.unpack_from("<H", data, at + 18)[0] == 224:                 # AMDGPU
            shoff, = struct.unpack_from("<Q", data, at + 40)
            size, count = struct.unpack_from("<HH", data, at + 58)
            for i in range(count):
                kind, = struct.unpack_from("<I", data, at + shoff + i * size + 4)
                if kind == 7:                                                 # notes
                    offset, = struct.unpack_from("<Q", data, at + shoff + i * size + 24)
                    n, d, _ = struct.unpack_from("<III", data, at + offset)
                    begin = at + offset + 12 + (n + 3) // 4 * 4
                    for k in msgpack.unpackb(data[begin:begin + d])["amdhsa.kernels"]:
                        yield k[".name"], k
        at = data.find(b"\x7fELF", at + 1)


def test_the_operators_kernels_keep_their_registers():
    """No kernel of the 8-bit cache, the log probabilities or the LM head has registers in scratch memory: 17 rows of the LM
    head took 136 us so, 110 without."""
    found = {n: k for n, k in kernels() if any(p in n for p in ("k_kv8_", "k_token_logprobs", "k_head_"))}
    assert all(any(p in n for n in found) for p in ("k_kv8_group", "k_token_logprobs_grad", "k_head_few"))
    spilled = {n: k[".private_segment_fixed_size"] for n, k in found.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]}
    assert not spilled
