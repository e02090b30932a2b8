"""The selective scan's kernels in the listing of what is built.  Their multiply-adds with an operand from another lane are written by hand, so the compiler keeps no
distance to them: along every path, what a matrix instruction (4 x 4 x 1, two passes) has written is read there four states later at the earliest, what a vector
instruction has written is read from other lanes two states later, and nothing that such an instruction writes is the addend of a matrix instruction one state
before it.  None of these kernels sets the execution mask by a vector comparison."""
import os
import re
import subprocess

import pytest

from listing_util import functions, registers
from paper_2407_12077_amd import build

MATRIX, OTHER_LANE = 4, 2


def states_of(text):
    op, _, rest = text.partition(" ")
    return int(rest.split()[0], 0) + 1 if op == "s_nop" else 1


def by_hand(text):
    return "row_newbcast" in text and not text.startswith("v_mov")


def reads_and_writes(text):
    op, _, rest = text.partition(" ")
    parts = re.split(r",\s*", re.sub(r"\s+row_newbcast.*", "", rest))
    return registers(" ".join(parts[1:])) | (registers(parts[0]) if "fmac" in op else set()), registers(parts[0]), registers(parts[1])


def walk(program, labels, start, budget, hit):
    """Calls hit(index, text) for every instruction fewer than `budget` states behind program[start], along every path."""
    todo, seen = [(start + 1, 0)], set()
    while todo:
        at, waited = todo.pop()
        while at < len(program) and waited < budget and (at, waited) not in seen:
            seen.add((at, waited))
            text = program[at][1]
            op = text.split()[0]
            hit(at, text)
            if op == "s_endpgm":
                break
            if op.startswith("s_cbranch"):
                todo.append((labels[text.split()[1]], waited + 1))
            elif op == "s_branch":
                at, waited = labels[text.split()[1]], waited + 1
                continue
            waited += states_of(text)
            at += 1


def too_early(program, labels):
    found = []
    for i, (line, text) in enumerate(program):
        op, _, rest = text.partition(" ")
        if op.startswith("v_mfma"):
            result, addend = registers(rest.split(",")[0]), registers(rest.split(",")[3])

            def after_matrix(at, now):
                if by_hand(now) and reads_and_writes(now)[0] & result:
                    found.append((line, program[at][0], "read"))
            walk(program, labels, i, MATRIX, after_matrix)

            def over_addend(at, now):
                if by_hand(now) and reads_and_writes(now)[1] & addend:
                    found.append((line, program[at][0], "overwritten"))
            walk(program, labels, i, 1, over_addend)
        elif op.startswith("v_") and not by_hand(text) and not op.startswith("v_cmp"):
            written = registers(rest.split(",")[0])
            if op.startswith("v_permlane") and "swap" in op:
                written = registers(rest)

            def from_lane(at, now):
                if by_hand(now) and reads_and_writes(now)[2] & written:
                    found.append((line, program[at][0], "from another lane"))
            walk(program, labels, i, OTHER_LANE, from_lane)
    return found


@pytest.mark.parametrize("source,kernels", [("selective_scan", ("scan_kernel", "scan_pieces_kernel")), ("selective_scan_backward", ("scan_backward_kernel",))])
def test_distances(tmp_path, source, kernels):
    out = str(tmp_path / "scan.s")
    subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, source + ".hip"), "-o", out], check=True, capture_output=True)
    found = {n: f for n, f in functions(open(out).read()).items() if any(k in n for k in kernels)}
    assert found and any(any(by_hand(t) for _, t in program) for program, _ in found.values())
    for name, (program, labels) in found.items():
        assert not any(t.startswith("v_cmpx") for _, t in program), name
        assert not too_early(program, labels), name


BAD = """
_Zone:
	v_mfma_f32_4x4x1_16b_f32 v[2:5], v6, v7, v[8:11] cbsz:4
	s_cbranch_scc1 .LBB0_2
	s_nop 7
.LBB0_2:
	s_nop 1
	v_mul_f32_dpp v1, v20, v2 row_newbcast:0 row_mask:0xf bank_mask:0xf
	s_endpgm
.Lfunc_end0:
"""


def test_the_walk_finds_what_is_too_early():
    program, labels = functions(BAD)["_Zone"]
    assert [f[2] for f in too_early(program, labels)] == ["read"]                   # along the branch: three states
    assert not too_early(*functions(BAD.replace("s_nop 1", "s_nop 2"))["_Zone"])
    assert [f[2] for f in too_early(*functions(BAD.replace("s_nop 1", "v_mov_b32_e32 v20, v21\n\ts_nop 2").replace("s_nop 2", "s_nop 0"))["_Zone"])].count("from another lane") == 1
    assert [f[2] for f in too_early(*functions(BAD.replace("s_cbranch_scc1 .LBB0_2\n\ts_nop 7\n.LBB0_2:\n\ts_nop 1", "v_mul_f32_dpp v8, v20, v30 row_newbcast:0 row_mask:0xf bank_mask:0xf\n\ts_nop 7")
                                                        )["_Zone"])] == ["overwritten"]
