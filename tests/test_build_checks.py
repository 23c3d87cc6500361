"""The build's look at the assembly: values that only some lanes move (CPU)."""
import pytest

from paper_2502_06798_amd.build_lib import masked_moves

SAVE, BACK = "\ts_and_saveexec_b64 s[0:1], vcc\n\ts_cbranch_execz .LBB0_2\n", ".LBB0_2:\n\ts_or_b64 exec, exec, s[0:1]\n"
TAIL = "\ts_endpgm\n"


@pytest.mark.parametrize("move", ["v_accvgpr_write_b32 a3, v17", "v_accvgpr_mov_b32 a3, a0", "scratch_store_dword off, v2, off offset:4"])
def test_moves_inside_a_branch_are_found(move):
    assert masked_moves(SAVE + f"; %bb.1:\n\t{move}   ; 4-byte Folded Spill\n" + BACK + TAIL) == [move]
    copied = "\ts_mov_b64 s[0:1], exec\n\ts_and_b64 s[2:3], s[0:1], vcc\n\ts_mov_b64 exec, s[2:3]\n\ts_cbranch_execz .LBB0_2\n"
    assert masked_moves(copied + f"\t{move}\n" + BACK + TAIL) == [move]
    other = SAVE.replace(".LBB0_2", ".LBB0_1") + ".LBB0_1:\n\ts_or_saveexec_b64 s[0:1], s[0:1]\n\ts_xor_b64 exec, exec, s[0:1]\n"
    assert masked_moves(other + f"\t{move}\n" + BACK + TAIL) == [move]                   # on the other side of it
    inner = SAVE + "\ts_and_saveexec_b64 s[4:5], s[6:7]\n\tv_add_f32_e32 v0, v0, v1\n\ts_or_b64 exec, exec, s[4:5]\n"
    assert masked_moves(inner + f"\t{move}\n" + BACK + TAIL) == [move]                   # after an inner one
    away = SAVE + "\ts_branch .LBB0_9\n" + BACK + TAIL + f".LBB0_9:\n\t{move}\n\ts_branch .LBB0_2\n"
    assert masked_moves(away) == [move]                                                  # placed behind the end


@pytest.mark.parametrize("move", ["v_accvgpr_write_b32 a3, v17", "scratch_store_dword off, v2, off offset:4"])
def test_moves_that_all_lanes_do_are_not(move):
    assert masked_moves(f"\t{move}\n" + SAVE + "\tglobal_store_dword v[0:1], v2, off\n" + BACK + f"\t{move}\n" + TAIL) == []
    assert masked_moves("\ts_cbranch_vccnz .LBB0_2\n" + f"\t{move}\n.LBB0_2:\n" + TAIL) == []    # a branch of whole waves
    loop = ".LBB0_1:\n" + SAVE + "\tv_mov_b32_e32 v0, v1\n" + BACK + "\ts_cbranch_scc0 .LBB0_1\n" + f"\t{move}\n" + TAIL
    assert masked_moves(loop) == []
    assert masked_moves(SAVE + "\tv_accvgpr_read_b32 v3, a17\n" + BACK + TAIL) == []     # out of one: a store's operand
