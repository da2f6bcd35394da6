"""Inline assembly, no GPU: a register that a statement writes by name is named among what it clobbers, or the compiler may keep something
of its own there."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1901_03040_amd", "csrc")
FILES = sorted(f for f in glob.glob(os.path.join(CSRC, "*")) if f.endswith((".h", ".hip", ".cpp")))


def statements(text):
    """The inline assembly statements of a source, each from its opening parenthesis to the closing one."""
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if c == '"' and text[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        yield text[m.end():i - 1]


def unnamed(statement):
    """Registers that the statement's instructions write by name and that it does not name as clobbered."""
    code = " ".join(re.findall(r'"((?:[^"\\]|\\.)*)"', statement.split(":")[0])).replace("\\n", "\n").replace("\\t", " ")
    written = {m for line in code.splitlines() for m in re.findall(r"^\s*\w+\s+(m0|vcc|exec|scc|[sv]\d+)\b", line)}
    last = statement.rsplit(":", 1)[-1] if statement.count(":") >= 3 else ""
    return written - set(re.findall(r'"(\w+)"', last))


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_registers_written_by_name_are_clobbered(path):
    with open(path) as f:
        for s in statements(f.read()):
            assert not unnamed(s), s


def test_the_check_itself():
    assert unnamed('"s_mov_b32 m0, %0\\n\\ts_nop 0" : : "s"(to) : "memory"') == {"m0"}
    assert unnamed('"s_mov_b32 m0, %0\\n\\ts_nop 0" : : "s"(to) : "m0", "memory"') == set()
    assert unnamed('"" ::: "memory"') == set()
    assert list(statements('x = asm_; asm volatile("a (" : "=v"(b) : "v"(c[0]));'))[0].startswith('"a ("')
