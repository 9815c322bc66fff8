"""Inline assembly declares the registers that it writes: m0, which the compiler may hold a value of its
own in, in the clobbers of every statement that names it as a destination."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2207_08867_amd", "csrc")


def statements(text):
    """The arguments of every asm(...) of a source, brackets balanced outside string literals."""
    for m in re.finditer(r"\basm\s*(?:volatile\s*)?\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if c == "\\" and quoted:
                i += 1
            elif c == '"':
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        yield text[m.end():i - 1]


def test_m0_is_declared():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path, encoding="utf-8") as f:
            for s in statements(f.read()):
                if re.search(r"s_\w+\s+m0\s*,", s):
                    seen += 1
                    assert '"m0"' in s, f"{os.path.basename(path)}: {s}"
    assert seen >= 2
