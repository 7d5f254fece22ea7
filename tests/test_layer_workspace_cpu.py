"""Workspace sizes of the layer operators (host functions, no GPU): a size asked for N tokens serves every
call of fewer, since the count of kept tokens changes with each draw of the cutoffs."""
import subprocess

import pytest
import torch

import ffn_plan
from paper_2606_29758_amd import layer

WIDTHS = [(3584, 14336), (1536, 6144), (1000, 4104), (64, 72), (8, 8), (8, 4096), (4096, 8), (2048, 800), (512, 1344),
          (568, 7952)]


def _counts():
    """Every count up to 300 tokens, then steps that meet every remainder of a tile, then around powers of two."""
    return sorted({*range(301), *range(301, 9000, 7), *range(9000, 70000, 131),
                   *(2 ** b + e for b in range(10, 20) for e in (-1, 1, 129))})


@pytest.mark.parametrize("d,f", WIDTHS)
@pytest.mark.parametrize("way", [dict(), dict(backward=True), dict(backward=True, preact=True)])
def test_ffn_workspace_never_falls(d, f, way):
    last, at = 0, 0
    for N in _counts():
        n = layer.gated_ffn_workspace_bytes(N, d, f, **way)
        assert n >= last, (at, N, last, n)
        last, at = n, N


def test_head_norm_workspace_never_falls():
    lib = layer.load()
    last = 0
    for N in _counts():
        n = lib.pspo_qk_norm_rope_workspace_bytes(N, 128)
        assert n >= last, N
        last = n


def test_plans_fit_the_workspace(tmp_path):
    """The slabs that the plans take, over many sizes, against the workspace's layout (host build of ffn_plan.h)."""
    exe = ffn_plan.build(tmp_path)
    run = subprocess.run([exe, "need"], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout + run.stderr


def test_no_size_for_widths_that_the_calls_refuse():
    for d, f in ((60, 72), (64, 70), (1, 8), (8, 4)):
        for way in (dict(), dict(backward=True), dict(backward=True, preact=True)):
            assert layer.gated_ffn_workspace_bytes(4, d, f, **way) == 0, (d, f, way)
    lib = layer.load()
    for D in (-8, 0, 4, 12, 520):
        assert lib.pspo_qk_norm_rope_workspace_bytes(4, D) == 0, D
    assert lib.pspo_qk_norm_rope_workspace_bytes(1 << 27, 128) == 0   # more tokens than a call takes


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses that no device call may touch")
def test_an_empty_call_takes_the_workspace_it_asked_for():
    """No tokens: 0 bytes are asked for, and the backward takes NULL for them (here up to the device check)."""
    lib = layer.load()
    A = 0x10000
    for flags, pre in ((512, None), (512 + 1024, A)):
        assert lib.pspo_gated_ffn_workspace_bytes(0, 64, 72, flags) == 0
        rc = lib.pspo_gated_ffn_bwd(None, None, A, A, A, pre, 0, 64, 72, 0, 0, None, A, A, A, None, 0, None)
        assert "null pointer" not in lib.pspo_last_error().decode(), (rc, lib.pspo_last_error())
    # with tokens it is asked for
    assert lib.pspo_gated_ffn_bwd(A, A, A, A, A, None, 4, 64, 72, 0, 0, A, A, A, A, None, 0, None) == 1
    assert "null pointer" in lib.pspo_last_error().decode()
