"""What a run cannot show of the kernels' sources: registers that inline
assembly uses are ones that the compiler knows of."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_14740_amd", "csrc")


def asm_statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r"\basm(?:\s+volatile)?\s*\(", text):
            depth, i = 1, m.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(text[i], 0)
                i += 1
            yield f"{os.path.basename(path)}:{text.count(chr(10), 0, m.start()) + 1}", text[m.end():i - 1]


def code_and_operands(body):
    """The strings of the template, and what follows its first colon outside them."""
    end = re.match(r'(?:\s*"(?:[^"\\]|\\.)*")+', body).end()
    return body[:end], body[end:]


STATEMENTS = list(asm_statements())


@pytest.mark.parametrize("where,body", STATEMENTS, ids=[w for w, _ in STATEMENTS])
def test_asm_declares_m0(where, body):
    """m0 is the compiler's to use between statements: assembly that writes it
    says so, and a load into LDS, which takes its place from m0, has it as an
    operand (or writes it itself)."""
    code, operands = code_and_operands(body)
    writes = re.search(r"\bs_\w+\s+m0\s*,", code)
    if writes:
        assert '"m0"' in operands, f"{where}: writes m0 and does not list it"
    if re.search(r"\blds\b", code):
        assert writes or '"{m0}"' in operands, f"{where}: m0 is not an operand"


def test_there_are_statements():
    assert any("lds" in code_and_operands(body)[0] for _, body in STATEMENTS)
