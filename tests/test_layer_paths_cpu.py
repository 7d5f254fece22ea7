"""The GPU tests' sizes reach every launch that the layer operators' plans choose (host builds of the plans)."""
import math
import os
import random
import subprocess

import pytest

import ffn_plan
import test_gpu_layer_ffn as elsewhere
from layer_sizes import DROP_PAST, FFN_PATHS, QK_PATHS
from paper_2606_29758_amd import build as pbuild


@pytest.fixture(scope="module")
def ffn_exe(tmp_path_factory):
    return ffn_plan.build(tmp_path_factory.mktemp("plan"))


def _ffn_launches(exe, sizes):
    """The launches of calls of these sizes: (product, tile, tile_n, ring, split along K)."""
    got = set()
    for i in range(0, len(sizes), 500):
        args = [str(v) for s in sizes[i:i + 500] for v in s]
        run = subprocess.run([exe, "cover", *args], capture_output=True, text=True, timeout=120)
        assert run.returncode == 0, run.stderr
        for line in run.stdout.splitlines():
            _, _, _, product, tile, tile_n, ring, parts = line.split()
            got.add((product, int(tile), int(tile_n), int(ring), int(parts) > 1))
    return got


def test_ffn_sizes_reach_every_launch(ffn_exe):
    rng = random.Random(3)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))   # noqa: E731
    sizes = [(log(1, 20000), 8 * log(1, 600), 8 * log(1, 2400)) for _ in range(40000)]
    reachable = _ffn_launches(ffn_exe, sizes)
    small = elsewhere.SIZES + [(2050, 1544, 3592), (4099, 3592, 2056)]   # compared in full
    tested = _ffn_launches(ffn_exe, small + FFN_PATHS)
    assert len(reachable) >= 45 and not reachable - tested, sorted(reachable - tested)
    # and each of the larger sizes is there for a launch that the small ones do not make
    assert _ffn_launches(ffn_exe, FFN_PATHS) - _ffn_launches(ffn_exe, small)


BYTES = dict(bf16=2, f32=4)


@pytest.fixture(scope="module")
def token_exe(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "token_plan_check")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "token_plan_check.cpp")
    res = subprocess.run([pbuild.hipcc(), "-O1", "-std=c++17", "-x", "c++", "-I", pbuild.CSRC, src, "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return exe


def _ask(exe, args):
    run = subprocess.run([exe, *args], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0
    return [tuple(int(v) for v in line.split()) for line in run.stdout.splitlines()]


def test_head_norm_sizes_reach_every_kernel(token_exe):
    got = _ask(token_exe, [f"qk:{N},{Hq},{Hk},{D},{BYTES[t]}" for N, Hq, Hk, D, _, _, t in QK_PATHS])
    for which in (3, 5):   # the forward's kernels, the backward's: lanes x past x type
        seen = {(g[0], g[which], s[6]) for g, s in zip(got, QK_PATHS)}
        assert seen == {(1 << i, p, t) for i in range(7) for p in (0, 1) for t in BYTES}, which
    for g, s in zip(got, QK_PATHS):
        assert g[1] >= 3, s                                          # passes of a wave, one after another
        assert g[4] >= 2 and s[0] % 4 != 0, s                        # tokens of a wave, a last work-group not full
    assert sum(g[2] for g in got) >= 14                              # queries and keys in one step of four passes
    assert any(g[1] > 4 and g[1] % 4 for g in got)                   # several steps, the last one not full


def test_dropout_sizes_go_past_the_caches(token_exe):
    got = _ask(token_exe, [f"drop:{N},{d},{BYTES[a] * (2 if r else 1) + BYTES[b]}" for N, d, a, b, r in DROP_PAST])
    assert all(lanes == 64 and past for lanes, past, _ in got)
    assert len({s[2:] for s in DROP_PAST}) == 6
