"""Compile-time guards for the layer's matrix-core kernels (CPU only: hipcc cross-compiles for gfx950).

Their MFMAs are inline asm on accumulators in place, whose latency the compiler does not know: any
copy or read of an accumulator needs its wait states behind the last MFMA, and the kernels may not
spill.  Checked in the assembly of every instantiation: no scratch memory, and no accumulator
register is read or moved within 20 wait states of an MFMA before it.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_29758_amd import build as pbuild


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("asm") / "ffn.s")
    cmd = [pbuild.hipcc(), *[f for f in pbuild.HIPCC_FLAGS if f != "-shared"], "-S", "--cuda-device-only",
           "-I", pbuild.INCLUDE, "-I", pbuild.CSRC, os.path.join(pbuild.CSRC, "ffn.hip"), "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    with open(out) as f:
        return f.read()


def _kernels(text):
    found = re.findall(r"^(_ZN4pspo\d+row_(?:gemm|jobs)_kernel\S*):\s.*?\n(.*?)\.Lfunc_end", text, re.S | re.M)
    assert len(found) >= 14
    return found


def test_no_scratch_memory(assembly):
    sizes = re.findall(r"^; ScratchSize: (\d+)", assembly, re.M)
    assert len(sizes) > 14 and set(sizes) == {"0"}
    spills = re.findall(r"\.vgpr_spill_count:\s*(\d+)", assembly)
    assert spills and set(spills) == {"0"}


def test_accumulators_are_read_behind_their_wait(assembly):
    for name, body in _kernels(assembly):
        lines = [x.strip() for x in body.splitlines()]
        lines = [x for x in lines if x and not x.startswith((";", "."))]
        waited, reads = None, 0
        for x in lines:
            if x.startswith("v_mfma"):
                assert re.match(r"v_mfma_f32_16x16x32_bf16 a\[(\d+:\d+)\], v\[\S+ v\[\S+ a\[\1\]", x), (name, x)
                waited = 0
            elif x.startswith("s_nop"):
                waited = None if waited is None else waited + int(x.split()[1]) + 1
            elif re.search(r"v_accvgpr_(read|mov)|\ba\[?\d", x) and not x.startswith("v_accvgpr_write"):
                reads += 1
                assert waited is None or waited >= 20, (name, x)
        assert reads > 0, name


def test_loads_wait_for_memory_by_count(assembly):
    """The waits for the loads in asm are the kernel's own; none of the compiler's waits for all loads stands
    between the MFMAs of a stage."""
    for name, body in _kernels(assembly):
        inside = body[body.index("v_mfma"):body.rindex("v_mfma")]
        own = len(re.findall(r"#ASMSTART\n\s*s_waitcnt vmcnt\(\d+\)", inside))
        every = len(re.findall(r"s_waitcnt vmcnt\(\d+\)", inside))
        jobs = "row_jobs" in name           # two loops, with an epilogue between them
        assert own >= 1 and (jobs or every == own), (name, own, every)
