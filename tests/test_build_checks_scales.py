"""The build's reading of the device assembly, scaled matrix instructions: their two scale registers are operands as well."""
import pytest

from paper_2501_16103_amd import build

MFMA = "v_mfma_scale_f32_32x32x64_f8f6f4 v[50:65], v[130:133], v[174:177], v[50:65], v20, v21 op_sel_hi:[1,0,0] cbsz:4 blgp:4"
BY_HAND = f"\t;;#ASMSTART\n\t{MFMA}\n\t;;#ASMEND\n"


def _kernel(body):
    return f"_ZN3moe12mx4_gemm_ldsEv:                  ; @kernel\n; %bb.0:\n{body}\ts_endpgm\n.Lfunc_end0:\n"


@pytest.mark.parametrize("register", ["v20", "v21", "v130", "v177", "v65"])
@pytest.mark.parametrize("between", ["", "\ts_nop 0\n"])
def test_an_operand_written_too_close_is_refused(register, between):
    with pytest.raises(RuntimeError, match="wait states behind"):
        build.check_mfma_operand_distance(_kernel(f"\tv_lshrrev_b32_e32 {register}, v3, v4\n{between}{BY_HAND}"))


@pytest.mark.parametrize("register", ["v20", "v21", "v130", "v177", "v65"])
def test_an_operand_written_early_enough_is_accepted(register):
    build.check_mfma_operand_distance(_kernel(f"\tv_lshrrev_b32_e32 {register}, v3, v4\n\ts_nop 1\n{BY_HAND}"))


def test_a_register_that_is_no_operand_is_accepted():
    build.check_mfma_operand_distance(_kernel("\tv_lshrrev_b32_e32 v22, v3, v4\n" + BY_HAND))


def test_a_scale_written_by_a_wide_move_is_refused():
    with pytest.raises(RuntimeError, match="wait states behind"):
        build.check_mfma_operand_distance(_kernel("\tv_mov_b64_e32 v[20:21], v[2:3]\n" + BY_HAND))
