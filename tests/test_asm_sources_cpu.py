"""Inline assembly names the registers that it writes."""

import glob
import os
import re

from paper_2608_15018_amd import build


def statements(text):
    """Each asm statement, up to its closing parenthesis."""
    for m in re.finditer(r"\basm\s+(?:volatile\s*)?\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            ch = text[i]
            if ch == '"' and text[i - 1] != "\\":
                quoted = not quoted
            depth += 0 if quoted else (ch == "(") - (ch == ")")
            i += 1
        yield text[m.start():i]


def test_statements_that_write_m0_say_so():
    seen = 0
    for path in glob.glob(os.path.join(build.CSRC, "*")):
        if os.path.isfile(path):
            with open(path) as f:
                text = f.read()
            for s in statements(text):
                if re.search(r"\bs_\w+ m0\b", s):
                    seen += 1
                    assert re.search(r':[^:]*"m0"[^:]*\)$', s), f"{os.path.basename(path)}: {s}"
    assert seen
