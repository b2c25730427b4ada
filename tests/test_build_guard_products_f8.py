"""The build refuses a library whose products of 8-bit floats move accumulators beside the matrix instructions that are written by hand, or hand them operands too late.

``build.check_products_f8`` reads the device assembly; here it is run on the real assembly and on copies of it with one mistake planted in each.
"""
import os
import re

import pytest

from paper_1803_03288_amd import build as b

KERNELS = pytest.mark.parametrize("key", b.ACCUMULATORS_F8)
MMA = r"^\s*(?:s_nop 1\n\s*)?v_mfma_"                # (with the wait that stands in front of it)


@pytest.fixture(scope="module")
def asm():
    return b.device_assembly(os.path.join(b.CSRC, "k9_product.hip"))


def planted(asm, key, at, line, group=0):
    """`line` in front of the first place where `at` (or a group of it) matches in the first of the kernels"""
    start = next(m.start() for m in re.finditer(r"^_Z\S*:", asm, re.M) if key in m.group(0))
    where = re.compile(at, re.M).search(asm, start).start(group)
    assert where < asm.index(".Lfunc_end", start)
    return asm[:where] + line + "\n" + asm[where:]


def first_operand(asm, key):
    start = next(m.start() for m in re.finditer(r"^_Z\S*:", asm, re.M) if key in m.group(0))
    return re.compile(r"v_mfma_\S+ a\[\d+:\d+\], v\[(\d+):").search(asm, start).group(1)


def test_generated_code_is_sound(asm):
    assert b.check_products_f8(asm) == []


@KERNELS
@pytest.mark.parametrize("line", ["\tv_accvgpr_read_b32 v1, a0", "\tv_accvgpr_write_b32 a0, v1", "\tv_accvgpr_mov_b32 a0, a1", "\tds_write_b128 v1, a[0:3]"])
def test_a_move_among_the_matrix_instructions_is_found(asm, key, line):
    assert any(key in x and "moved among" in x for x in b.check_products_f8(planted(asm, key, MMA, line)))


@KERNELS
@pytest.mark.parametrize("line", ["\tv_accvgpr_read_b32 v1, a0", "\tds_write_b128 v1, a[0:3]", "\tglobal_store_dwordx4 v[2:3], a[0:3], off"])
def test_a_read_before_the_wait_is_found(asm, key, line):
    bad = b.check_products_f8(planted(asm, key, r"^\s*s_nop 15", ".LBB_planted:\n" + line))
    assert any(key in x and "before the wait" in x for x in bad)


@KERNELS
def test_a_spill_is_found(asm, key):
    assert any(key in x and "spills" in x for x in b.check_products_f8(planted(asm, key, MMA, "\tscratch_store_dword off, v1, s32")))


@KERNELS
@pytest.mark.parametrize("between", ["", "\n\ts_nop 0"])
def test_an_operand_written_right_before_is_found(asm, key, between):
    line = f"\tv_mov_b32_e32 v{first_operand(asm, key)}, 0{between}"
    assert any(key in x and "right before" in x for x in b.check_products_f8(planted(asm, key, r"^\s*(v_mfma_)", line, 1)))


@KERNELS
def test_an_operand_written_two_waits_before_is_sound(asm, key):
    line = f"\tv_mov_b32_e32 v{first_operand(asm, key)}, 0\n\ts_nop 1"
    assert b.check_products_f8(planted(asm, key, r"^\s*(v_mfma_)", line, 1)) == []


def test_an_operand_written_before_a_branch_is_found():
    key = b.ACCUMULATORS_F8[0]
    text = f"_Z{key}v:\n.LA:\n\tv_mfma_x a[0:3], v[0:7], v[8:15], a[0:3], v20, v21\n\tv_mov_b32_e32 v20, 0\n\ts_cbranch_scc1 .LA\n\ts_endpgm\n.Lfunc_end0:\n"
    assert any("right before" in x for x in b.check_operands(text, key))
    assert b.check_operands(text.replace("\ts_cbranch", "\ts_nop 0\n\ts_cbranch"), key) == []


@KERNELS
def test_a_renamed_kernel_is_found(asm, key):
    assert f"no kernel {key} found" in b.check_products_f8(asm.replace(key, key.replace("product", "produce")))
