"""Inline-assembly loads from global memory stand behind bounds checks.  An asm statement that is not volatile counts as a
pure function of its operands, which a compiler may move or run ahead of the check; so each of them has to be volatile."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_36959_b200", "csrc")


def test_global_loads_in_assembly_are_volatile():
    seen = 0
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r'\basm\s*(volatile)?\s*\(\s*((?:"[^"]*"\s*)+)', text):
            if re.search(r"\bld(\.volatile|\.relaxed[.\w]*|\.acquire[.\w]*)?\.global|\bld\.[\w.]*global|\bmultimem\.ld", m.group(2)):
                seen += 1
                assert m.group(1), (os.path.basename(path), m.group(2)[:60])
    assert seen >= 2
