"""The build's reading of the device assembly, the layer for few tokens and the 4-bit products: no register spill in the loop over k, whose
loads are steps ahead, and no array left in memory."""
import pytest

from paper_2501_16103_amd import build

MFMA = "\tv_mfma_f32_16x16x16_bf16 v[0:3], v[10:11], v[20:21], v[0:3]\n"
LOAD = "\tscratch_load_dword v5, off, off offset:16\n"


NAMES = {"_ZN3moe13few_tokens_upINS_7FewBf16ELi1EEEvNS_7FewArgsE": 8, "_ZN3moe13mx4_gemm_rowsILi1EEEvNS_11Mx4GemmArgsE": 4}   # MFMAs of a k-step


def _kernel(name, prologue="", tile="", k=""):
    """A loop over tiles around a loop over k."""
    mfmas = NAMES[name]
    return (f"{name}:      ; @kernel\n; %bb.0:\n{prologue}.LBB0_1:\n{tile}.LBB0_2:\n{k}{MFMA * mfmas}"
            "\ts_cbranch_scc1 .LBB0_2\n\ts_barrier\n\ts_cbranch_scc1 .LBB0_1\n\ts_endpgm\n.Lfunc_end0:\n")


@pytest.mark.parametrize("name", NAMES)
def test_a_spill_in_the_k_loop_is_refused(name):
    with pytest.raises(RuntimeError, match="register spill inside a k loop"):
        build.check_no_spill_in_k_loops(_kernel(name, k=LOAD))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("where", ["prologue", "tile"])
def test_spills_around_it_are_accepted(where, name):
    build.check_no_spill_in_k_loops(_kernel(name, **{where: LOAD}))
    build.check_no_spill_in_k_loops(_kernel(name))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("size,ok", [(124, True), (324, False)])
def test_arrays_in_memory(size, ok, name):
    text = _kernel(name) + f"    .name:           {name}\n    .private_segment_fixed_size: {size}\n"
    if ok:
        build.check_no_spill_in_k_loops(text)
    else:
        with pytest.raises(RuntimeError, match="private memory"):
            build.check_no_spill_in_k_loops(text)
