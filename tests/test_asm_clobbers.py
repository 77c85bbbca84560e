"""Assembly in the kernels' sources that sets m0 or loads into LDS says so in its clobber list.  No GPU: the sources are read."""
import glob
import os
import re

from paper_2506_15724_amd import build as B


def statements(text):
    """Every asm statement, up to the parenthesis that closes it (none stands in its strings)."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if c == '"' and text[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        yield text[m.start():i]


def test_what_the_compiler_cannot_see_is_listed():
    found = 0
    for path in sorted(glob.glob(os.path.join(B.CSRC, "*.h")) + glob.glob(os.path.join(B.CSRC, "*.hip"))):
        for s in statements(open(path).read()):
            code = s.split('"')[1]
            listed = re.findall(r'"([^"]*)"', s)[1:]
            if re.search(r"\bm0\b", code):
                found += 1
                assert "m0" in listed, (path, s)
            if re.search(r"load_lds|\blds\b", code):
                assert "memory" in listed, (path, s)
    assert found >= 4
