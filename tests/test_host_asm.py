"""CPU check of the kernels' inline assembler: a scalar register that an instruction writes by name is named in the clobbers too, since the
compiler may hold a value of its own there, and a load to LDS gets its place through m0 as an operand."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_08888_amd", "csrc")


def statements(text):
    """(template, operands, clobbers) of every asm statement."""
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
        yield parts[0], "".join(parts[1:3]), parts[3] if len(parts) > 3 else ""


def missing(template, operands, clobbers):
    """Scalar registers that the template writes and the clobbers do not name, or that it reads without getting them."""
    written = re.findall(r"(?:^|\W|\\[nt])s_(?!waitcnt|nop)\w+\s+(m0|vcc|exec|s\d+)\b", template)
    reads = ["m0"] if "_load_lds" in template and "m0" not in written else []
    return [r for r in written if f'"{r}"' not in clobbers] + [r for r in reads if f'"{{{r}}}"' not in operands]


def test_the_check_itself():
    one = 'asm volatile("s_mov_b32 m0, %0\\n\\tnext" ::"s"(at(1)) : "memory");'
    two = 'asm volatile("s_mov_b32 m0, %0\\n\\tnext" ::"s"(at[1]) : "memory", "m0");  // asm("s_mov_b32 m0, 0")'
    assert [missing(*s) for s in statements(one + two)] == [["m0"], []]
    three = 'asm volatile("s_nop 0\\n\\tglobal_load_lds_dword %1, off" ::"{m0}"(at), "v"(from) : "memory");'
    assert [missing(*s) for s in statements(three + three.replace("{m0}", "s"))] == [[], ["m0"]]
    assert [missing(*s) for s in statements('asm("s_waitcnt vmcnt(0)" : "+v"(x)); asm volatile("");')] == [[], []]


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*"))), ids=os.path.basename)
def test_assembler_names_what_it_writes(path):
    with open(path) as f:
        for statement in statements(f.read()):
            assert not missing(*statement), statement[0]
