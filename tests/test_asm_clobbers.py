"""Inline assembly names the registers that it writes without an operand: the compiler keeps values in them otherwise (CPU only)."""
import os
import re

from paper_2204_08211_amd import build as hip_build


def statements(text):
    """The arguments of every asm statement: its text, and what follows the text."""
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(", text):
        at, depth = m.end(), 1
        while depth:
            quoted = re.compile(r'"(?:[^"\\]|\\.)*"').match(text, at)
            at = quoted.end() if quoted else at + 1
            depth += 0 if quoted else {"(": 1, ")": -1}.get(text[at - 1], 0)
        parts = re.match(r'\s*((?:"(?:[^"\\]|\\.)*"\s*)+)(.*)\)$', text[m.end():at], re.S)
        yield parts.group(1), parts.group(2)


def test_registers_written_in_assembly_are_named():
    written = 0
    for name in sorted(os.listdir(hip_build.CSRC)):
        with open(os.path.join(hip_build.CSRC, name)) as f:
            for code, operands in statements(f.read()):
                for register in re.findall(r"\b(?:s|v)_\w+\s+(m0|vcc|exec|scc|s\[?\d+|v\[?\d+)\b", code):
                    written += 1
                    assert f'"{register}"' in operands.split(":")[-1], (name, code)
    assert written >= 1
