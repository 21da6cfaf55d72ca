"""Kernels of the 8-bit contraction and of the step between halves are written to a register budget too: the build refuses spills."""
import pytest

from paper_2605_17633_amd import build


@pytest.mark.parametrize("name", ["_Z19gemm_i8_wide_kernelILi64ELi64ELi2ELi0EEv10GemmI8Args13GemmTileRange", "_Z23gemm_i8_wide_cut_kernelILi256ELi256ELi1ELi2ELi0EEv10GemmI8Args13GemmTileRange",
                                  "_ZN12_GLOBAL__N_129residual_norm_backward_kernelILi3ELi64ELb1ELb1ELb1EEEvNS_8BackArgsE", "_ZN12_GLOBAL__N_120residual_norm_kernelILi1ELi16ELb1ELNS_7StepOutE1EEEvNS_8StepArgsE"])
def test_spills_of_8_bit_contractions_and_steps_are_refused(name):
    assert build.spilled([{"name": name, "VGPRs Spill": 1}]) and not build.spilled([{"name": name, "VGPRs Spill": 0}])
