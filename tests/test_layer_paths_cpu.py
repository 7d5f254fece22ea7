"""The GPU tests' sizes reach every launch that the layer operators' plans choose (host builds of the plans)."""
import math
import random
import subprocess

import pytest

import ffn_plan
import test_gpu_layer_ffn as elsewhere
from layer_sizes import FFN_PATHS


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
