"""Inline assembly names the registers that it writes beside its operands."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_01676_amd", "csrc")


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if not os.path.isfile(path):
            continue
        text = open(path, encoding="utf-8").read()
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
            depth, at, quoted = 1, m.end(), False
            while depth:
                c = text[at]
                if quoted:
                    at += c == "\\"
                    quoted = c != '"' or text[at - 1:at + 1] == '\\"'
                elif c == '"':
                    quoted = True
                else:
                    depth += (c == "(") - (c == ")")
                at += 1
            yield os.path.basename(path), text[m.end():at - 1]


def parts(statement):
    """(template, clobbers): the text before the first colon outside of quotes, and after the third"""
    fields = re.split(r':(?=(?:[^"]*"[^"]*")*[^"]*$)', statement)
    return fields[0], fields[3] if len(fields) > 3 else ""


@pytest.mark.parametrize("register", ["m0", "vcc", "exec", "scc"])
def test_written_registers_are_declared(register):
    seen = 0
    for name, statement in statements():
        template, clobbers = parts(statement)
        # (an instruction's first operand is what it writes)
        if re.search(rf"\b[sv]_\w+\s+{register}(_lo|_hi)?\b", template):
            seen += 1
            assert f'"{register}"' in clobbers, f"{name}: asm({statement}) writes {register}"
    assert seen or register != "m0"


def test_statements_are_found():
    found = list(statements())
    assert len(found) >= 10 and any("s_mov_b32 m0" in parts(s)[0] for _, s in found)
    assert parts('"a: b" :: "s"(x) : "memory", "m0"') == ('"a: b" ', ' "memory", "m0"')
