"""Inline assembly of the kernels' sources: what a block writes by name, it
declares. The compiler may otherwise keep a value of its own in that register
across the block."""
import glob
import os
import re

import pytest

from paper_2111_04867_amd import build

# registers that instructions name, and the suffixes of their halves
NAMED = ("m0", "vcc", "exec", "flat_scratch")
WRITES = re.compile(r"^\s*(?:s_|v_)\w+\s+(%s)(?:_lo|_hi)?\b" % "|".join(NAMED))
COMPARES = re.compile(r"^\s*v_cmpx?_\w+\s+(vcc|exec)\b")


def blocks(text):
    """Every asm statement's text, between its parentheses."""
    for m in re.finditer(r"\basm\s+(?:volatile\s*)?\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            ch = text[at]
            if ch == '"' and text[at - 1] != "\\":
                quoted = not quoted
            depth += (ch == "(") - (ch == ")") if not quoted else 0
            at += 1
        yield text[m.end():at - 1]


def undeclared(block):
    """Registers that the instructions write and the clobbers do not name."""
    parts, depth, quoted, start = [], 0, False, 0
    for i, ch in enumerate(block):
        if ch == '"' and block[i - 1] != "\\":
            quoted = not quoted
        if quoted:
            continue
        depth += (ch in "([") - (ch in ")]")
        if ch == ":" and not depth:
            parts.append(block[start:i])
            start = i + 1
    parts.append(block[start:])
    code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', parts[0]))
    code = code.replace("\\n", "\n").replace("\\t", " ")
    declared = set(re.findall(r'"(\w+)"', parts[3])) if len(parts) > 3 else set()
    wrote = {m[1] for line in code.split("\n") for m in [WRITES.match(line) or COMPARES.match(line)]
             if m}
    return sorted(wrote - declared)


SOURCES = sorted(glob.glob(os.path.join(build.CSRC, "*.h")) +
                 glob.glob(os.path.join(build.CSRC, "*.hip")))


@pytest.mark.parametrize("source", SOURCES, ids=os.path.basename)
def test_named_registers_are_declared(source):
    with open(source) as f:
        for block in blocks(f.read()):
            assert not undeclared(block), block


def test_the_audit_finds_an_undeclared_register():
    written = r'"s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(p), "s"(q)'
    assert undeclared(written + r' : "memory"') == ["m0"]
    assert undeclared(written) == ["m0"]
    assert undeclared(written + r' : "memory", "m0"') == []
    assert undeclared(r'"s_waitcnt vmcnt(%0)" ::"n"(3) : "memory"') == []
    assert undeclared(r'"v_cmp_eq_u32 vcc, %0, %1" : : "v"(a[i]), "v"(b) : "memory"') == ["vcc"]
