"""Inline assembly tells the compiler of m0, which it may use itself (CPU)."""

import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_18239_amd", "csrc")
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith((".hip", ".hpp")))


def statements(text):
    """The asm statements of a file, each to its closing bracket."""
    for m in re.finditer(r"\basm\s*(volatile\s*)?\(", text):
        depth, quoted, i = 1, False, m.end()
        while depth:
            c = text[i]
            quoted ^= c == '"' and text[i - 1] != "\\"
            depth += 0 if quoted else (c == "(") - (c == ")")
            i += 1
        yield text[m.start():i]


def test_the_reader():
    text = 'asm volatile("s_mov_b32 m0, %0\\n\\tx %1" : : "s"(f(a)), "v"(b)); y; asm("")'
    assert list(statements(text)) == ['asm volatile("s_mov_b32 m0, %0\\n\\tx %1" : : "s"(f(a)), "v"(b))', 'asm("")']


@pytest.mark.parametrize("name", SOURCES)
def test_m0_is_named_where_it_is_written(name):
    text = open(os.path.join(CSRC, name)).read()
    for s in statements(text):
        if re.search(r"\bm0\s*,", s):
            assert re.search(r':[^:]*"m0"[^:]*\)$', s), s
