"""The build's scan for instructions whose operands the register allocator takes for undefined."""
from paper_2504_00030_amd import isa_guard

BAD = """
name:            _ZN2sd1kEv
body:             |
  bb.70:
    renamable $vgpr71 = nofpexcept V_FMA_F32_e64 0, $vgpr106, 0, $sgpr20, 1, $vgpr115, 0, 0, implicit $mode, implicit $exec
    renamable $vgpr106 = nofpexcept V_EXP_F32_e32 killed $vgpr71, implicit $mode, implicit $exec
    renamable $vgpr30_vgpr31_vgpr32_vgpr33 = contract V_MFMA_F32_16X16X4F32_vgprcd_e64 $vgpr70, $vgpr106, killed $vgpr30_vgpr31_vgpr32_vgpr33, 0, 0, 0, implicit $mode, implicit $exec
    renamable $vgpr26_vgpr27_vgpr28_vgpr29 = contract V_MFMA_F32_16X16X4F32_vgprcd_e64 undef $vgpr71, $vgpr106, killed $vgpr26_vgpr27_vgpr28_vgpr29, 0, 0, 0, implicit $mode, implicit $exec
    renamable $vgpr5 = V_PERM_B32_e64 $vgpr6, undef renamable $vgpr7, killed $sgpr4, implicit $exec
    renamable $agpr0_agpr1_agpr2_agpr3 = V_MFMA_F32_16X16X32_BF16_e64 $vgpr8_vgpr9_vgpr10_vgpr11, undef $agpr4_agpr5_agpr6_agpr7, $agpr0_agpr1_agpr2_agpr3, 0, 0, 0, implicit $mode, implicit $exec
"""

GOOD = """
name:            _ZN2sd1kEv
body:             |
  bb.70:
    undef renamable $vgpr70 = IMPLICIT_DEF
    renamable $vgpr4_vgpr5_vgpr6_vgpr7 = V_MFMA_F32_16X16X32_BF16_vgprcd_e64 $vgpr70_vgpr71_vgpr72_vgpr73, $vgpr8_vgpr9_vgpr10_vgpr11, 0, 0, 0, 0, implicit $mode, implicit $exec
    undef renamable $vgpr8 = V_MOV_B32_e32 0, implicit $exec, implicit-def $vgpr8_vgpr9
    $sgpr0 = S_MOV_B32 undef $sgpr1
"""


def test_flags_operands_taken_for_undefined():
    msgs = isa_guard.undefined_operands(BAD.splitlines())
    assert len(msgs) == 3 and all(m.startswith("_ZN2sd1kEv") for m in msgs)
    assert all(x in m for x, m in zip(("undef $vgpr71", "undef renamable $vgpr7", "undef $agpr4"), msgs))


def test_accepts_defined_operands():
    assert isa_guard.undefined_operands(GOOD.splitlines()) == []


def test_refuses_a_print_without_functions():
    assert len(isa_guard.undefined_operands("\tv_mov_b32 v0, v1\n".splitlines())) == 1
