"""Inline assembly names every fixed register that it writes, so that the compiler keeps
nothing of its own there."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_16308_amd", "csrc")
WRITES = re.compile(r"\b[sv]_\w+\s+(m0|vcc(?:_lo|_hi)?|exec(?:_lo|_hi)?|[sv]\d+|[sv]\[\d+:\d+\])\s*,")


def statements(text):
    """(template, clobbers) of each asm statement."""
    for at in re.finditer(r"\basm\s+volatile\s*\(|\basm\s*\(", text):
        depth, i, quoted = 1, at.end(), False
        parts, last = [], at.end()
        while depth:
            c = text[i]
            if quoted:
                i += c == "\\"
                quoted = c != '"'
            elif c == '"':
                quoted = True
            elif c in "([{":
                depth += 1
            elif c in ")]}":
                depth -= 1
            elif c == ":" and depth == 1:
                # ("::" leaves out a part; a qualified name stands in brackets)
                parts.append(text[last:i])
                last = i + 1
            i += 1
        parts.append(text[last:i - 1])
        yield parts[0], parts[3] if len(parts) > 3 else ""


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith((".hip", ".hpp", ".cpp", ".h"))))
def test_written_registers_are_named(name):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for template, clobbers in statements(text):
        for reg in WRITES.findall(template.replace("\\n", " ").replace("\\t", " ")):
            assert f'"{reg}"' in clobbers, f"{name}: {template.strip()} writes {reg}"


def test_statements_are_found():
    got = list(statements('asm volatile("s_mov_b32 m0, %0\\n\\tx %1, %2" ::"s"(f(a ? b : c)), "v"(o) : "m0", "memory");  asm("v_nop");'))
    assert len(got) == 2 and '"m0"' in got[0][1] and WRITES.findall(got[0][0]) == ["m0"] and got[1] == ('"v_nop"', "")
