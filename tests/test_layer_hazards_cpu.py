"""Compile-time guard for the wait states that the compiler does not see in the row products (CPU only).

Their matrix instructions and loads into LDS are inline asm, which the compiler's hazard rules pass over: a vector
instruction that writes an operand of a matrix instruction has to stand two wait states before it, one that writes
a scalar register five before a load that reads it, and m0 one before the load.  Checked in the assembly of every
kernel of ffn.hip.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_29758_amd import build as pbuild


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("asm") / "ffn.s")
    cmd = [pbuild.hipcc(), *[f for f in pbuild.HIPCC_FLAGS if f != "-shared"], "-S", "--cuda-device-only",
           "-I", pbuild.INCLUDE, "-I", pbuild.CSRC, os.path.join(pbuild.CSRC, "ffn.hip"), "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    with open(out) as f:
        text = f.read()
    found = {}
    for name, body in re.findall(r"^(_ZN4pspo\S*kernel\S*):\s.*?\n(.*?)\.Lfunc_end", text, re.S | re.M):
        lines = [x.split(";")[0].strip() for x in body.splitlines()]
        found[name] = [x for x in lines if x and not x.startswith(".")]
    assert len(found) >= 25
    return found


def _regs(text, kind):
    out = set()
    for m in re.finditer(r"\b%s\[(\d+):(\d+)\]|\b%s(\d+)\b" % (kind, kind), text):
        out |= set(range(int(m.group(1)), int(m.group(2)) + 1)) if m.group(1) else {int(m.group(3))}
    return out


def _written(line):
    """The destination of an instruction."""
    parts = line.split(None, 1)
    return parts[1].split(",")[0] if len(parts) > 1 else ""


def _near(lines, i, states, wrong):
    """An instruction less than `states` wait states before lines[i] that `wrong` finds."""
    waited, j = 0, i - 1
    while j >= 0 and waited < states:
        if wrong(lines[j]):
            return lines[j]
        waited += int(lines[j].split()[1]) + 1 if lines[j].startswith("s_nop") else 1
        j -= 1
    return None


def _vector(line):
    return line.startswith("v_") and not line.startswith(("v_mfma", "v_cmp"))


def _faults(lines):
    for i, x in enumerate(lines):
        if x.startswith("v_mfma"):
            ops = x.split(None, 1)[1].split(",")
            v, a = _regs(",".join(ops[1:3]), "v"), _regs(ops[3], "a")
            found = _near(lines, i, 2, lambda y: _vector(y) and (_regs(_written(y), "v") & v or _regs(_written(y), "a") & a))
            if found:
                yield x, found
        elif x.startswith("buffer_load") and x.endswith("lds"):
            s = _regs(x, "s")
            for found in (_near(lines, i, 5, lambda y: y.startswith("v_") and (_regs(_written(y), "s") & s
                                                                              or _written(y) == "m0")),
                          _near(lines, i, 1, lambda y: y.startswith("s_") and _written(y) == "m0")):
                if found:
                    yield x, found


def test_operands_stand_before_their_instructions(kernels):
    loads = mfmas = 0
    for name, lines in kernels.items():
        assert not list(_faults(lines)), (name, next(_faults(lines)))
        loads += sum(x.startswith("buffer_load") and x.endswith("lds") for x in lines)
        mfmas += sum(x.startswith("v_mfma") for x in lines)
    assert loads > 300 and mfmas > 900


def test_the_check_finds_what_it_is_for():
    mfma = "v_mfma_f32_16x16x32_bf16 a[0:3], v[8:11], v[12:15], a[0:3]"
    load = "buffer_load_dwordx4 v3, s[4:7], s9 offen lds"
    assert list(_faults(["v_mov_b32_e32 v9, v1", "s_nop 0", mfma]))
    assert not list(_faults(["v_mov_b32_e32 v9, v1", "s_nop 1", mfma]))
    assert list(_faults(["v_accvgpr_write_b32 a2, 0", mfma]))
    assert list(_faults(["v_readfirstlane_b32 s9, v1", "s_nop 3", load]))
    assert not list(_faults(["v_readfirstlane_b32 s9, v1", "s_nop 4", load]))
    assert list(_faults(["s_mov_b32 m0, s3", load]))
    assert not list(_faults(["s_mov_b32 m0, s3", "s_nop 0", load]))
