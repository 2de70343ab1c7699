"""CPU check of the kernels' inline assembler: a register that an instruction names by itself is named in the clobbers too, since the
compiler may hold a value of its own there."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_08888_amd", "csrc")


def statements(text):
    """(template, clobbers) of every asm statement."""
    text = re.sub(r"//[^\n]*", "", text)
    for start in re.finditer(r"\basm\s*(?:volatile\s*)?\(", text):
        depth, parts, at, quoted = 1, [""], start.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            if not quoted:
                depth += (c in "([") - (c in ")]")
                if c == ":" and depth == 1:
                    parts.append("")
                    at += 1
                    continue
            parts[-1] += c if depth else ""
            at += 1
        yield parts[0], parts[3] if len(parts) > 3 else ""


def missing(template, clobbers):
    """Scalar registers that the template's instructions write and the clobbers do not name."""
    written = re.findall(r"\bs_\w+\s+(m0|vcc|exec|s\d+)\b", template)
    return [r for r in written if f'"{r}"' not in clobbers]


def test_the_check_itself():
    one = 'asm volatile("s_mov_b32 m0, %0\\n\\tnext" ::"s"(at(1)) : "memory");'
    two = 'asm volatile("s_mov_b32 m0, %0\\n\\tnext" ::"s"(at[1]) : "memory", "m0");  // asm("s_mov_b32 m0, 0")'
    assert [missing(*s) for s in statements(one + two)] == [["m0"], []]
    assert [missing(*s) for s in statements('asm("s_waitcnt vmcnt(0)" : "+v"(x)); asm volatile("");')] == [[], []]


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*"))), ids=os.path.basename)
def test_assembler_names_what_it_writes(path):
    with open(path) as f:
        for template, clobbers in statements(f.read()):
            assert not missing(template, clobbers), template
