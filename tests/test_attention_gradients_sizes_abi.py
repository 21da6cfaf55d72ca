"""Sizes of windows that the gradient of attention takes because the forward call does, without a GPU: it gets as far as the workspace, the last check."""
import pytest

from paper_2605_17633_amd import binding as B
from test_attention_gradients_abi import call


@pytest.mark.parametrize("sizes", [dict(row_stride=8 * 1000 * 1000), dict(row_stride=1 << 40, S=1, w=1), dict(groups=1 << 22, h=16, S=16, w=4, row_stride=1024, grad_stride=1024),
                                   dict(groups=1 << 20, h=12, S=196, w=14, row_stride=768, grad_stride=768, mask_block=128)])
def test_windows_that_are_far_apart_or_many(sizes):
    assert call(**sizes, ws_bytes=16) == B.EWORKSPACE


@pytest.mark.parametrize("sizes", [dict(row_stride=8 * 1000 * 1000), dict(groups=1 << 21, h=16, row_stride=1024, grad_stride=1024)])
def test_grids_are_refused(sizes):
    assert call(**{**dict(S=256, w=16, mask_block=128), **sizes}) == B.EUNSUPPORTED


@pytest.mark.parametrize("S,w", [(1, 1), (49, 7), (196, 14)])
@pytest.mark.parametrize("d", [16, 80])
def test_workspace_of_windows(S, w, d):
    """What a window's walks hand to each other stays in LDS: only the sums of the tables' gradients need memory, those of 256 workgroups at most."""
    for groups, h in ((1, 1), (25, 12), (100, 16), (1 << 20, 16)):
        assert B.ssam_sparse_attention_backward_workspace_bytes(groups, S, w, h, d) == min(groups * h, 256) * 2 * 32 * d * 4
