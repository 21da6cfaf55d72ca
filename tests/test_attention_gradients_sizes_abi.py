"""Sizes that the gradient of attention asks for, without a GPU."""
import pytest

from paper_2605_17633_amd import binding as B


@pytest.mark.parametrize("S,w", [(1, 1), (49, 7), (196, 14)])
@pytest.mark.parametrize("d", [16, 80])
def test_workspace_of_windows(S, w, d):
    """What a window's walks hand to each other stays in LDS: only the sums of the tables' gradients need memory, those of 256 workgroups at most."""
    for groups, h in ((1, 1), (25, 12), (100, 16), (1 << 20, 16)):
        assert B.ssam_sparse_attention_backward_workspace_bytes(groups, S, w, h, d) == min(groups * h, 256) * 2 * 32 * d * 4
