"""The head-decay kernels' accumulators on their way into LDS, in the listing of what is built: whatever way the compiler arranged the blocks, every path from a
matrix product to an LDS write of its result has the wait states that the product takes: eight behind one of four passes (16 x 16 x 32 bf16), ten behind
an fp32 one of eight."""
import os
import subprocess

from listing_util import early_lds_writes, functions
from paper_2407_12077_amd import build

STATES = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}


def test_no_accumulator_is_written_to_lds_early(tmp_path):
    out = str(tmp_path / "head_decay.s")
    subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "head_decay.hip"), "-o", out], check=True, capture_output=True)
    kernels = {n: f for n, f in functions(open(out).read()).items() if "mix_kernel" in n}
    assert len(kernels) == 7 and sum(any(t.startswith("ds_write_b128") for _, t in program) for program, _ in kernels.values()) == 5
    for name, (program, labels) in kernels.items():
        assert {t.split()[0] for _, t in program if t.startswith("v_mfma")} <= set(STATES)
        assert not early_lds_writes(program, labels, STATES), name


MERGED = """
_Zone:
	s_cbranch_scc1 .LBB0_2
	v_mfma_f32_16x16x32_bf16 v[2:5], v[6:9], v[10:13], v[2:5]
	s_nop 11
	s_branch .LBB0_3
.LBB0_2:
	v_mfma_f32_16x16x32_bf16 v[2:5], v[6:9], v[10:13], v[2:5]
	s_nop 3
.LBB0_3:
	ds_write_b128 v1, v[2:5]
	s_endpgm
.Lfunc_end0:
"""


def test_the_walk_follows_branches():
    """Two products whose LDS write has been merged: one path waits long enough, the other one does not."""
    program, labels = functions(MERGED)["_Zone"]
    assert [(b, c) for _, b, c in early_lds_writes(program, labels, STATES)] == [(11, 4)]
    program, labels = functions(MERGED.replace("s_nop 3", "s_nop 11"))["_Zone"]
    assert not early_lds_writes(program, labels, STATES)
    reused = MERGED.replace("s_nop 3", "v_mov_b32_e32 v2, 0\n\tv_mov_b32_e32 v3, 0\n\tv_mov_b32_e32 v4, 0\n\tv_mov_b32_e32 v5, 0")
    assert not early_lds_writes(*functions(reused)["_Zone"], STATES)
