"""Inline assembly says which registers it writes besides its operands: the compiler keeps values in all others across it.  No GPU needed."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_12707_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h")))


def statements(text):
    """(instructions, what stands behind them) of every asm statement."""
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            depth += 0 if quoted else (c == "(") - (c == ")")
            at += 1
        body = text[m.end():at - 1]
        strings = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', body)
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', strings.group(1))), body[strings.end():]


@pytest.mark.parametrize("source", SOURCES, ids=os.path.basename)
def test_special_registers_that_are_written_are_named(source):
    for instructions, behind in statements(open(source).read()):
        for line in instructions.split("\\n\\t"):
            name, _, operands = line.strip().partition(" ")
            written = operands.split(",")[0].strip()
            if written in ("m0", "vcc"):
                assert '"%s"' % written in behind, (instructions, behind)
            if name.startswith("s_cmp_"):
                assert '"scc"' in behind, (instructions, behind)
        # all lanes are active again behind it, as they were before
        changes = re.findall(r"\S+ exec, (\S+?)(?:\\n|$)", instructions)
        assert not changes or changes[-1] == "-1", instructions


def test_there_is_such_assembly():
    found = [text for source in SOURCES for text, _ in statements(open(source).read())]
    assert any("m0" in text for text in found) and any("s_cmp_" in text for text in found)
