"""Inline assembly names the registers that it writes besides its operands: the compiler may keep
something in them otherwise."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = sorted(glob.glob(os.path.join(ROOT, "paper_2308_15152_amd", "csrc", "*"))
                 + glob.glob(os.path.join(ROOT, "include", "**", "*.h*"), recursive=True))
# a literal register as the first operand of an instruction: v_..., s_... or ..., not a store
WRITES = re.compile(r"(?:^|\\n\\t|\\n|\s)(?:s|v)_\w+\s+((?:m0|vcc|exec|scc|[sv]\d+|[sv]\[\d+:\d+\]))\b")


def statements(text):
    """(template, clobbers) of every asm statement."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        body = text[m.end():at - 1]
        literal = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)*)', body).group(1)
        parts = re.split(r"::|:", re.sub(r'"(?:[^"\\]|\\.)*"', lambda s: s.group().replace(":", ";"),
                                         body[len(literal):]))
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', literal)), parts[-1]


def written_unnamed(text):
    return [(template, register) for template, clobbers in statements(text)
            for register in WRITES.findall(template) if f'"{register}"' not in clobbers]


@pytest.mark.parametrize("path", [os.path.relpath(p, ROOT) for p in SOURCES])
def test_written_registers_are_named(path):
    with open(os.path.join(ROOT, path)) as f:
        assert written_unnamed(f.read()) == []


def test_the_check_itself():
    head = 'asm volatile("s_mov_b32 m0, %2\\n\\ts_nop 0\\n\\tglobal_load %0, %1" ::"v"(off[i]), "s"(a ? b : c)'
    assert written_unnamed(head + ' : "memory");') == [
        ("s_mov_b32 m0, %2\\n\\ts_nop 0\\n\\tglobal_load %0, %1", "m0")]
    assert written_unnamed(head + ' : "m0", "memory");') == []
    assert written_unnamed('asm volatile("v_add %0, %1" : "+v"(x) : "v"(y));') == []
