"""Inline assembly names the special registers that it writes (read from the sources, no GPU)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_14787_amd", "csrc")
FILES = sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h")))


def statements(text):
    """(line, body) of every asm statement: from its parenthesis to the one that closes it, strings left alone."""
    for m in re.finditer(r"\basm\s+volatile\s*\(|\basm\s*\(", text):
        depth, at = 1, m.end()
        while depth:
            if text[at] == '"':
                at = re.compile(r'(?:[^"\\]|\\.)*"').match(text, at + 1).end()
                continue
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        yield text.count("\n", 0, m.start()) + 1, text[m.end():at - 1]


def code_of(body):
    """The instructions: the string literals before the first colon outside of one."""
    out, at = [], 0
    for m in re.finditer(r'\s*"((?:[^"\\]|\\.)*)"', body):
        if m.start() != at:
            break
        out.append(m.group(1))
        at = m.end()
    return "".join(out).replace("\\n", "\n").replace("\\t", " "), body[at:]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_m0_is_named(path):
    for line, body in statements(open(path).read()):
        code, operands = code_of(body)
        if re.search(r"^\s*s_\w+\s+m0\b", code, re.M):
            assert '"m0"' in operands.split(":")[-1], f"{os.path.basename(path)}:{line}"


def test_the_reading_itself():
    text = 'x; asm volatile("s_mov_b32 m0, %0\\n\\t" "s_nop 0" ::"s"(f(a)), "v"(b) : "memory"); asm volatile("" : "+v"(c)); asm("s_add_u32 m0, m0, 4" ::: "m0");'
    found = [(code_of(b)[0], '"m0"' in code_of(b)[1].split(":")[-1]) for _, b in statements(text)]
    assert [f[1] for f in found] == [False, False, True] and found[0][0].startswith("s_mov_b32 m0") and found[1][0] == ""
