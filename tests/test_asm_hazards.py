"""Wait states around the stores that the kernels issue in inline assembly.

The compiler keeps dependent instructions of gfx950 apart where the hardware
does not, but it does not look into assembly blocks. For a 16-byte store in one
that leaves two rules to the source: a matrix instruction of 8 passes has to be
12 wait states behind before the store reads its result, and after the store 2
have to pass before its registers are written. Both have to come from waits
that the source itself places (s_nop within a block); how far apart the
compiler's other instructions happen to keep them does not count.

The sources are compiled here with the library's own flags (no GPU needed).
"""
import os
import re
import shutil

import pytest

from paper_2111_04867_amd import build

BEFORE, AFTER = 12, 2
STORE = re.compile(r"^global_store_dwordx[34] ")


def registers(operand):
    """Numbers of v[a:b] or va."""
    m = re.match(r"v\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"v(\d+)$", operand)
    return {int(m[1])} if m else set()


def states(line):
    """Wait states of an s_nop, else 0."""
    return 1 + int(line.split()[1], 0) if line.startswith("s_nop ") else 0


def faults(asm):
    """(stores in assembly blocks, those without their waits)."""
    product = {}  # register: wait states that blocks placed since a product wrote it
    stores, bad, block = 0, [], None
    for line in asm.split("\n"):
        line = line.strip()
        if line.startswith(";;#ASMSTART"):
            block = []
        elif line.startswith(";;#ASMEND"):
            for i, t in enumerate(block):
                for r in product:
                    product[r] += states(t)
                if STORE.match(t):
                    stores += 1
                    data = registers(t.split()[2].rstrip(","))
                    behind = sum(states(u) for u in block[i + 1:])
                    if behind < AFTER or any(product.get(r, BEFORE) < BEFORE for r in data):
                        bad.append(t)
            block = None
        elif not line or line[0] in ".;":
            continue
        elif block is not None:
            block.append(line)
        elif re.match(r"^_Z\w+:", line):
            product = {}
        elif line.startswith("v_"):
            wrote = registers(line.split()[1].rstrip(","))
            for r in wrote:
                product.pop(r, None)
                if line.startswith("v_mfma"):
                    product[r] = 0
    return stores, bad


@pytest.mark.parametrize("source", ["ffn.hip", "tokens.hip"])
def test_stores_have_their_waits(source, tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc is not installed")
    out = tmp_path / "out.s"
    p = build.device_asm(os.path.join(build.CSRC, source), str(out))
    err = p.communicate()[1]
    assert p.returncode == 0, err[-2000:]
    stores, bad = faults(out.read_text())
    assert not bad, (len(bad), bad[:3])
    assert stores > 0 or source == "tokens.hip"


def test_the_audit_finds_what_is_missing():
    def one(*lines):
        return len(faults("\n".join(lines))[1])

    product, start, end = "v_mfma_f32_16x16x32_bf16 v[2:5], v[8:11], v[12:15], v[2:5]", \
        ";;#ASMSTART", ";;#ASMEND"
    store = [start, "global_store_dwordx4 v[14:15], v[2:5], off sc1", "s_nop 1", end]
    assert one(product, *store) == 1
    assert one(product, start, "s_nop 10", end, *store) == 1
    assert one(product, start, "s_nop 11", end, *store) == 0
    assert one(product, start, "s_nop 11", end, product, *store) == 1
    assert one(product, "v_mov_b32_e32 v2, v9", start, "s_nop 11", end, *store) == 0
    assert one(*store) == 0
    assert one(store[0], store[1], "s_nop 0", end) == 1
