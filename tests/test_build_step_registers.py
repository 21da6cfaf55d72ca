"""Registers of the step between halves, as the build records them: two waves to a SIMD, but for the two kernels that are written for one."""
import pytest

from test_build_resources import recorded

ALONE = "residual_norm_backward_kernelILi4ELi64ELb%dELb1ELb1E"       # rows above 1536, with or without a norm behind the branch, with the second LayerNorm and the weights' gradients


def test_gradients():
    found = [(n, r) for n, r in recorded() if "residual_norm_backward_kernelI" in n]
    assert len(found) == 48                                          # six widths, either norm or none, with the weights' gradients or without
    for name, r in found:
        alone = any(ALONE % post in name for post in (0, 1))
        assert r["spill"] == 0 and r["scratch"] == 0 and r["vgprs"] + r["agprs"] <= (512 if alone else 256) and r["occupancy"] >= (1 if alone else 2), (name, r)


@pytest.mark.parametrize("kernel,count", [("residual_norm_kernelI", 36), ("quantize_rows_kernelI", 8)])
def test_forward(kernel, count):
    """Bound by the requests in flight: four waves to a SIMD at least"""
    found = [(n, r) for n, r in recorded() if kernel in n]
    assert len(found) == count
    for name, r in found:
        assert r["spill"] == 0 and r["vgprs"] + r["agprs"] <= 128, (name, r)
