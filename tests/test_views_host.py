"""The host's test whether strided views share a byte (csrc/evo_views.h), against sets of bytes: never "apart" of views
that share one, and "apart" of every two views of one packed buffer that do not."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def apart(tmp_path_factory):
    d = tmp_path_factory.mktemp("views")
    src, lib = d / "views.cpp", d / "views.so"
    src.write_text('#include "evo_views.h"\nextern "C" int apart(const evo::View *a, const evo::View *b) {\n'
                   '    return evo::views_apart(*a, *b);\n}\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC",
                    "-I", os.path.join(ROOT, "paper_2404_11068_amd", "csrc"), "-o", str(lib), str(src)], check=True)
    f = ctypes.CDLL(str(lib)).apart

    def call(a, b):
        A, B = ((ctypes.c_int64 * 6)(*x) for x in (a, b))
        return bool(f(A, B))
    return call


def _bytes(v):
    at, row, tok, n, length, block = v
    return {at + i * row + j * tok + c for i in range(n) for j in range(length) for c in range(block)}


def test_never_apart_where_bytes_are_shared(apart):
    rng = random.Random(1)
    seen = [0, 0, 0]
    for _ in range(60000):
        def view():
            block = rng.randint(1, 6)
            tok, n, length = rng.choice([0, rng.randint(1, 20)]), rng.randint(1, 4), rng.randint(1, 4)
            row = rng.choice([0, rng.randint(1, 60), tok * length, tok * length + rng.randint(0, 9), tok * rng.randint(1, 5)])
            return (rng.randint(1000, 1080), row, tok, n, length, block)
        a, b = view(), view()
        if rng.random() < 0.5:
            b = (b[0], a[1], a[2]) + b[3:]
        shared = bool(_bytes(a) & _bytes(b))
        says = apart(a, b)
        assert not (says and shared), (a, b)
        assert says == apart(b, a), (a, b)
        seen[2 if shared else 1 if says else 0] += 1
    assert seen[1] > 1000 and seen[2] > 1000


def test_views_of_a_packed_buffer(apart):
    """Blocks of one token side by side, rows with or without room behind them, tokens or rows outermost, views from any
    token on and of any lengths: exactly where they share no byte."""
    rng = random.Random(2)
    for _ in range(20000):
        parts = [rng.randint(1, 5) for _ in range(rng.randint(2, 4))]
        width, rows, length = sum(parts) + rng.choice([0, 0, 3]), rng.randint(1, 4), rng.randint(1, 6)
        tok, row = (width, width * length + rng.choice([0, 0, 1, 5])) if rng.random() < 0.7 else (width * rows, width)

        def view(i):
            first = rng.randint(0, length - 1) if rng.random() < 0.3 else 0
            n, l = rows, rng.choice([length - first, rng.randint(1, length - first)])
            # the stride of an axis of one entry says nothing
            r, t = (row if n > 1 else rng.choice([row, 0, 7])), (tok if l > 1 else rng.choice([tok, parts[i], 0]))
            return (5000 + first * tok + sum(parts[:i]), r, t, n, l, parts[i])
        a, b = view(rng.randrange(len(parts))), view(rng.randrange(len(parts)))
        assert apart(a, b) == (not _bytes(a) & _bytes(b)), (a, b)
    # blocks that reach into the next one's place
    assert not apart((0, 64, 16, 4, 4, 8), (6, 64, 16, 4, 4, 8)) and not apart((0, 64, 16, 4, 4, 8), (10, 64, 16, 4, 4, 8))
    assert apart((0, 64, 16, 4, 4, 8), (8, 64, 16, 4, 4, 8))
    # far apart in size: strides of more than 2^32
    far = 1 << 40
    assert apart((1 << 44, far, far >> 10, 8, 1024, 64), ((1 << 44) + 64, far, far >> 10, 8, 1024, 64))
    assert not apart((1 << 44, far, far >> 10, 8, 1024, 64), ((1 << 44) + 63, far, far >> 10, 8, 1024, 64))
