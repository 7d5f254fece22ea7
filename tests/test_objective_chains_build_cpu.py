"""Compile-time guards for every kernel of objective.hip that holds the row products' inline asm, chains of tiles and
products of one launch among them (CPU only: hipcc cross-compiles for gfx950).

The rules are those of test_layer_hazards_cpu.py and test_layer_build_cpu.py: an operand of a matrix instruction is
written two wait states before it at least, a scalar register of a load into LDS five, m0 one, and an accumulator is read
twenty behind the last matrix instruction.  Here they are followed backwards along every way through a kernel, jumps
included: a chain goes from a tile's epilogue, past the zeroing of its accumulators, back to the first matrix
instruction of the loop.
"""
import os
import re
import shutil
import subprocess

import pytest

import test_layer_hazards_cpu as hazards
from paper_2606_29758_amd import build as pbuild

KINDS = ("row_gemm_kernel", "row_chain_kernel", "row_jobs_kernel")


class Flow:
    """A kernel's instructions, and those that may run right before each."""

    def __init__(self, body):
        self.lines, labels, jumps = [], {}, []
        for x in body.splitlines():
            x = x.split(";")[0].strip()
            label = re.match(r"(\.L\w+):", x)
            if label:
                labels[label.group(1)] = len(self.lines)
            elif x and not x.startswith("."):
                if x.startswith(("s_branch", "s_cbranch")):
                    jumps.append((len(self.lines), x.split()[-1]))
                self.lines.append(x)
        self.before = [[i - 1] if i and not self.lines[i - 1].startswith(("s_branch", "s_endpgm", "s_setpc")) else []
                       for i in range(len(self.lines))]
        for at, label in jumps:
            if labels[label] < len(self.lines):
                self.before[labels[label]].append(at)

    def near(self, i, states, wrong):
        """An instruction less than `states` wait states before lines[i], on some way there, that `wrong` finds."""
        seen, todo = {}, [(j, 0) for j in self.before[i]]
        while todo:
            j, waited = todo.pop()
            if waited >= states or seen.get(j, states) <= waited:
                continue
            seen[j] = waited
            x = self.lines[j]
            if wrong(x):
                return x
            waited += int(x.split()[1]) + 1 if x.startswith("s_nop") else 1
            todo += [(k, waited) for k in self.before[j]]
        return None

    def faults(self):
        regs, written = hazards._regs, hazards._written
        for i, x in enumerate(self.lines):
            if x.startswith("v_mfma"):
                ops = x.split(None, 1)[1].split(",")
                v, a = regs(",".join(ops[1:3]), "v"), regs(ops[3], "a")
                yield x, self.near(i, 2, lambda y: hazards._vector(y) and (regs(written(y), "v") & v or regs(written(y), "a") & a))
            elif x.startswith("buffer_load") and x.endswith("lds"):
                s = regs(x, "s")
                yield x, self.near(i, 5, lambda y: y.startswith("v_") and (regs(written(y), "s") & s or written(y) == "m0"))
                yield x, self.near(i, 1, lambda y: y.startswith("s_") and written(y) == "m0")
            elif self.reads_accumulators(x):
                yield x, self.near(i, 20, lambda y: y.startswith("v_mfma"))

    @staticmethod
    def reads_accumulators(x):
        parts = x.split(None, 1)
        if len(parts) < 2 or not x.startswith(("v_accvgpr_read", "v_accvgpr_mov", "global_store", "buffer_store", "ds_write")):
            return False
        return bool(hazards._regs(parts[1], "a"))


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("asm") / "objective.s")
    cmd = [pbuild.hipcc(), *[f for f in pbuild.HIPCC_FLAGS if f != "-shared"], "-S", "--cuda-device-only",
           "-I", pbuild.INCLUDE, "-I", pbuild.CSRC, os.path.join(pbuild.CSRC, "objective.hip"), "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    with open(out) as f:
        text = f.read()
    found = {name: Flow(body) for name, body in re.findall(r"^(_ZN4pspo\S*kernel\S*):\s.*?\n(.*?)\.Lfunc_end", text, re.S | re.M)
             if any(k in name for k in KINDS)}
    for kind, least in zip(KINDS, (10, 5, 4)):
        assert sum(kind in name for name in found) >= least, kind
    return found


def test_wait_states_on_every_way(kernels):
    for name, flow in kernels.items():
        assert [f for f in flow.faults() if f[1]] == [], name
        assert any(flow.reads_accumulators(x) for x in flow.lines), name
        assert sum(x.startswith("v_mfma") for x in flow.lines) >= 16 and any(x.endswith("lds") for x in flow.lines), name


def test_matrix_instructions_add_in_place(kernels):
    for name, flow in kernels.items():
        for x in flow.lines:
            if x.startswith("v_mfma"):
                assert re.match(r"v_mfma_f32_16x16x32_bf16 a\[(\d+:\d+)\], v\[\S+ v\[\S+ a\[\1\]", x), (name, x)


def test_a_chain_goes_back_to_its_loop(kernels):
    """What the ways are followed for: some accumulator is zeroed on a way that jumps back before the matrix
    instructions that add to it."""
    for name, flow in kernels.items():
        if "row_chain" not in name:
            continue
        zeroed = [i for i, x in enumerate(flow.lines) if x.startswith("v_accvgpr_write")]
        mfmas = [i for i, x in enumerate(flow.lines) if x.startswith("v_mfma")]
        back = [i for i, x in enumerate(flow.lines) if x.startswith(("s_branch", "s_cbranch"))
                and any(i in flow.before[j] and j <= mfmas[0] for j in range(mfmas[0] + 1))]
        assert zeroed and any(i > mfmas[-1] for i in back), name


def test_the_check_finds_what_it_is_for():
    mfma, zero = "v_mfma_f32_16x16x32_bf16 a[0:3], v[8:11], v[12:15], a[0:3]", "v_accvgpr_write_b32 a2, 0"
    load, read = "buffer_load_dwordx4 v3, s[4:7], s9 offen lds", "v_accvgpr_read_b32 v1, a0"
    found = lambda *x: any(f[1] for f in Flow("\n".join(x)).faults())   # noqa: E731
    loop = (".LBB0_1:", mfma, "s_nop 15", "s_nop 3", read, "s_cbranch_scc1 .LBB0_2")
    assert found(*loop, zero, "s_branch .LBB0_1", ".LBB0_2:", "s_endpgm")
    assert not found(*loop, zero, "s_nop 0", "s_branch .LBB0_1", ".LBB0_2:", "s_endpgm")
    assert found(".LBB0_1:", read, mfma, "s_cbranch_scc1 .LBB0_1", "s_endpgm")
    assert not found(".LBB0_1:", read, mfma, "s_nop 15", "s_nop 2", "s_cbranch_scc1 .LBB0_1", "s_endpgm")
    assert found("v_readfirstlane_b32 s9, v1", "s_cbranch_scc1 .LBB0_1", "s_nop 4", ".LBB0_1:", load, "s_endpgm")
    assert found("s_mov_b32 m0, s3", ".LBB0_1:", load, "s_endpgm")
    assert not found("v_readfirstlane_b32 s9, v1", "s_branch .LBB0_1", load, ".LBB0_1:", "s_endpgm")
