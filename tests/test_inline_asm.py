"""What the kernels' inline assembly changes is what it says that it changes."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = sorted(f for pat in ("*.hip", "*.hpp")
               for f in glob.glob(os.path.join(ROOT, "paper_2505_17701_amd", "csrc", pat)))


def statements(text):
    """(instructions, what follows them) of each asm statement"""
    for m in re.finditer(r"\basm(?:\s+volatile)?\s*\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if c == '"' and text[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        body = re.match(r'((?:\s*"(?:[^"\\]|\\.)*")*)(.*)', text[m.end():i - 1], re.S)
        yield body.group(1), body.group(2)


@pytest.mark.parametrize("path", FILES, ids=[os.path.basename(f) for f in FILES])
def test_a_statement_that_writes_m0_names_it(path):
    with open(path) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for code, rest in statements(text):
        if re.search(r"\bs_\w+\s+m0\b", code):
            assert re.search(r'"m0"', rest), code


def test_some_statement_writes_m0():
    """(the scan finds what it looks for)"""
    text = 'asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 4" ::"s"(a(b)) : "memory");'
    (code, rest), = statements(text)
    assert re.search(r"\bs_\w+\s+m0\b", code) and '"m0"' not in rest
