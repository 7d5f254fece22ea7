"""Inline asm of the kernels names what it writes beside its operands (source check, CPU only)."""
import glob
import os
import re

import pytest

from paper_2606_29758_amd import build as pbuild

SOURCES = sorted(glob.glob(os.path.join(pbuild.CSRC, "*.h")) + glob.glob(os.path.join(pbuild.CSRC, "*.hip")))


def _statements(text):
    """Every asm statement, from its opening parenthesis to the closing one."""
    for m in re.finditer(r"\basm(?:\s+volatile)?\s*\(", text):
        depth, i, quoted = 1, m.end(), False
        while depth:
            c = text[i]
            if c == '"' and text[i - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            i += 1
        yield text[m.end():i - 1]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_registers_written_by_name_are_clobbered(path):
    """m0, vcc, exec or scc as a destination inside the text needs the compiler to know."""
    with open(path) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for s in _statements(text):
        code = s[:s.index('"', 1 + s.index('"')) + 1] if '"' in s else s
        clobbers = s.rsplit(":", 1)[-1] if ":" in s else ""
        for line in re.split(r"\\n(?:\\t)?", code.strip('" ')):
            m = re.match(r"\s*[sv]_\w+\s+(m0|vcc|exec)\b", line)
            assert m is None or f'"{m.group(1)}"' in clobbers, s.strip()


def test_the_check_finds_what_it_is_for():
    bad = 'asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0" : : "s"(x) : "memory");'
    (s,) = _statements(bad)
    assert "m0" in s and '"m0"' not in s.rsplit(":", 1)[-1]
