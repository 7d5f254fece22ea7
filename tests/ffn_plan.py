"""Compiles tests/ffn_plan_check.cpp, which asks ffn_plan.h how the gated block's products are launched."""
import os
import subprocess

from paper_2606_29758_amd import build as pbuild

HERE = os.path.dirname(os.path.abspath(__file__))


def build(folder) -> str:
    exe = os.path.join(str(folder), "ffn_plan_check")
    cmd = [pbuild.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++17", "-x", "hip", "-I", pbuild.INCLUDE,
           "-I", pbuild.CSRC, os.path.join(HERE, "ffn_plan_check.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return exe
