"""What the inline assembly of the token rows' products writes, it declares."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2008_00325_amd", "csrc")


def statements(text):
    """The arguments of each asm statement."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        yield text[m.end():at - 1]


def test_assembly_that_writes_m0_says_so():
    found = 0
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".hip", ".hpp")):
            continue
        for s in statements(open(os.path.join(CSRC, name)).read()):
            if re.search(r"s_mov_b32 m0", s):
                found += 1
                assert re.search(r':\s*"m0"\s*,\s*"memory"\s*$|:\s*"memory"\s*,\s*"m0"\s*$', s), f"{name}: {s}"
    assert found
