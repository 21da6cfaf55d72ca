"""Sizes of the gradient of attention: what its workspace is used for."""
import pytest
import torch

import test_gpu_attention_gradients as T
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16


@pytest.mark.parametrize("case", [(1, 1, 1, 16, 32, 1.0, "position", False), (3, 14, 5, 64, 32, 0.5, "content", True), (17, 14, 16, 80, 32, 0.4, "position", False), (40, 7, 12, 32, 32, 0.5, "content", False),
                                  (2, 14, 3, 80, 128, 0.4, "content", False), (2, 15, 3, 32, 128, 0.5, "position", False), (3, 33, 3, 64, 128, 0.4, "content", True)])
def test_workspace_is_enough(case):
    """A workspace of the size that is asked for, inside a larger buffer: the same bits as with one that the binding makes, and nothing beside it is touched."""
    announce("sparse_attention_backward workspace", case)
    groups, w, h, d, tile, r, order, drop = case
    (qkv, rel, sigma, out_rows, dout, out), want = T.run(case, seed=33)
    n = B.ssam_sparse_attention_backward_workspace_bytes(groups, w * w, w, h, d)
    around = torch.full((n + 8192,), 0x5a, dtype=torch.uint8, device=DEV)
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, dout, out_rows=out_rows, workspace=around[4096:4096 + n])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool((around[:4096] == 0x5a).all()) and bool((around[4096 + n:] == 0x5a).all())
