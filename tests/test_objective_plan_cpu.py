"""The objectives' plans against their workspace, over many sizes (host build of objective_plan.h, CPU only)."""
import os
import shutil
import subprocess

import pytest

from paper_2606_29758_amd import build as pbuild

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="hipcc not available")
def test_plans_fit_the_workspace(tmp_path):
    exe = str(tmp_path / "objective_plan_check")
    cmd = [pbuild.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++17", "-x", "hip", "-I", pbuild.INCLUDE,
           "-I", pbuild.CSRC, os.path.join(HERE, "objective_plan_check.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout + run.stderr
