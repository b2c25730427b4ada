"""The build refuses a library whose largest products move accumulators beside the matrix instructions that are written by hand.

``build.check_accumulators`` reads the device assembly; here it is run on the real assembly and on copies of it with one mistake planted in each.
"""
import os
import re

import pytest

from paper_1803_03288_amd import build as b

KEY = b.ACCUMULATORS


@pytest.fixture(scope="module")
def asm():
    return b.device_assembly(os.path.join(b.CSRC, "k8_product.hip"))


def planted(asm, at, line):
    """`line` in front of the first place where `at` matches in the first of the kernels"""
    start = next(m.start() for m in re.finditer(r"^_Z\S*:", asm, re.M) if KEY in m.group(0))
    where = re.compile(at, re.M).search(asm, start).start()
    assert where < asm.index(".Lfunc_end", start)
    return asm[:where] + line + "\n" + asm[where:]


def test_generated_code_leaves_the_accumulators_where_they_are(asm):
    assert b.check_accumulators(asm) == []


@pytest.mark.parametrize("line", ["\tv_accvgpr_read_b32 v1, a0", "\tv_accvgpr_write_b32 a0, v1", "\tv_accvgpr_mov_b32 a0, a1"])
def test_a_move_among_the_matrix_instructions_is_found(asm, line):
    bad = b.check_accumulators(planted(asm, r"^\s*v_mfma_", line))
    assert any(KEY in x and "moved among" in x for x in bad)


def test_a_read_before_the_wait_is_found(asm):
    bad = b.check_accumulators(planted(asm, r"^\s*s_nop 15", ".LBB_planted:\n\tv_accvgpr_read_b32 v1, a0"))
    assert any(KEY in x and "before the wait" in x for x in bad)


def test_a_spill_is_found(asm):
    bad = b.check_accumulators(planted(asm, r"^\s*v_mfma_", "\tscratch_store_dword off, v1, s32"))
    assert any(KEY in x and "spills" in x for x in bad)


def test_a_renamed_kernel_is_found(asm):
    assert b.check_accumulators(asm.replace(KEY, "18product_kernel_257")) == [f"no kernel {KEY} found"]
