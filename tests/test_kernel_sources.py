"""Rules that the kernels' sources keep to, read from the sources."""
import glob
import os
import re

from paper_2609_03494_amd import build


def _statements(text):
    """Every inline assembly statement, from its parenthesis to the one that closes it."""
    for at in re.finditer(r"\b(?:__asm__|asm)\s+volatile\s*\(", text):
        depth, i = 1, at.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        yield text[at.end():i]


def test_assembly_names_the_scalar_registers_that_it_writes():
    """A register that a statement's text sets by name is among its clobbers: the compiler may keep something in it."""
    found = 0
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*"))):
        for s in _statements(open(path).read()):
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', s.split(" : ")[0]))
            clobbers = set(re.findall(r'"(\w+)"', s.rsplit(":", 1)[-1]))
            for reg in re.findall(r"\bs_mov_b(?:32|64)\s+(m0|vcc\w*|exec\w*|s\d+|s\[\d+:\d+\])", code):
                found += 1
                assert reg in clobbers, (os.path.basename(path), s)
    assert found
