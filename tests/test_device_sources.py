"""Inline assembly of the device code tells the compiler what it changes (read from the sources; no GPU)."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _blocks():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_1705_01598_amd", "csrc", "*.h*"))):
        text = open(path).read()
        for start in re.finditer(r"\basm\s+volatile\s*\(|\basm\s*\(", text):
            depth, at = 1, start.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(text[at], 0)
                at += 1
            yield os.path.basename(path), text[start.end():at - 1]


def test_assembly_leaves_m0_to_the_compiler():
    """A block that needs a value in m0 takes it as an operand: written inside, the compiler would not know."""
    found = 0
    for name, block in _blocks():
        assert not re.search(r"\bm0\s*,", block), (name, block)
        found += '"{m0}"' in block
    assert found
