"""Compile-time guards for the objectives' kernels (CPU only: hipcc cross-compiles for gfx950): those of the layer's
row products, which they share, in the assembly of objective.hip."""
import os
import re
import shutil
import subprocess

import pytest

import test_layer_build_cpu as build_checks
import test_layer_hazards_cpu as hazard_checks
from paper_2606_29758_amd import build as pbuild


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("asm") / "objective.s")
    cmd = [pbuild.hipcc(), *[f for f in pbuild.HIPCC_FLAGS if f != "-shared"], "-S", "--cuda-device-only",
           "-I", pbuild.INCLUDE, "-I", pbuild.CSRC, os.path.join(pbuild.CSRC, "objective.hip"), "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    with open(out) as f:
        return f.read()


def test_no_scratch_memory(assembly):
    build_checks.test_no_scratch_memory(assembly)



def test_accumulators_are_read_behind_their_wait(assembly, monkeypatch):
    found = re.findall(r"^(_ZN4pspo\d+row_gemm_kernel\S*):\s.*?\n(.*?)\.Lfunc_end", assembly, re.S | re.M)
    assert len(found) >= 10
    monkeypatch.setattr(build_checks, "_kernels", lambda text: found)
    build_checks.test_accumulators_are_read_behind_their_wait(assembly)
    build_checks.test_loads_wait_for_memory_by_count(assembly)


def test_operands_stand_before_their_instructions(assembly):
    loads = mfmas = 0
    for name, body in re.findall(r"^(_ZN4pspo\S*kernel\S*):\s.*?\n(.*?)\.Lfunc_end", assembly, re.S | re.M):
        lines = [x.split(";")[0].strip() for x in body.splitlines()]
        lines = [x for x in lines if x and not x.startswith(".")]
        if "row_gemm" not in name:   # the compiler's own instructions keep its own rules
            continue
        assert not list(hazard_checks._faults(lines)), (name, next(hazard_checks._faults(lines)))
        loads += sum(x.startswith("buffer_load") and x.endswith("lds") for x in lines)
        mfmas += sum(x.startswith("v_mfma") for x in lines)
    assert loads > 150 and mfmas > 500
