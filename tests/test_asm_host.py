"""Inline assembly of the kernels names the special registers that it writes (source check, no GPU)."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _statements():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2404_11068_amd", "csrc", "*"))):
        text = open(path).read()
        for m in re.finditer(r"\basm volatile\s*\(", text):
            depth, i = 1, m.end()
            while depth:
                if text[i] == '"':
                    i = text.index('"', i + 1)
                depth += {"(": 1, ")": -1}.get(text[i], 0)
                i += 1
            yield os.path.basename(path), text[m.end():i - 1]


def test_m0_is_named_where_it_is_written():
    writes = 0
    for name, body in _statements():
        code = re.match(r'(\s*"[^"]*")+', body).group(0)
        if re.search(r"s_mov_b32 m0\b", code):
            writes += 1
            assert '"m0"' in body[len(code):], (name, body)
    assert writes >= 2
