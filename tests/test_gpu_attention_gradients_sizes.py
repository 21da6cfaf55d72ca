"""Gradients of attention in windows whose rows lie further apart than 32 bits reach, and in more (group, head) than a grid of workgroups would hold: the bits of the ordinary calls."""
import ctypes as C
import math

import pytest
import torch

import test_gpu_attention_gradients as T
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16


@pytest.mark.parametrize("d,tile", [(64, 32), (80, 32), (16, 128)])
def test_rows_far_apart(d, tile):
    """196 rows of 11.2 MB: 2.2 GB a window, of both the features and their gradients."""
    announce("sparse_attention_backward rows far apart", d, tile)
    groups, w, h = 2, 14, 2
    S, row = w * w, 5600 * 1000
    (qkv, rel, sigma, _, dout, out), (want, wh, ww) = T.run((groups, w, h, d, tile, 0.5, "content", False), seed=31)
    src, dst = (torch.full((groups * S, row), math.nan, dtype=BF, device=DEV) for _ in range(2))
    at = [8, row // 2, row - h * d]                                   # places of q, k, v in a row
    for i in range(3):
        src[:, at[i]:at[i] + h * d] = qkv[:, :, i].reshape(groups * S, h * d)
    dh, dw = torch.empty_like(rel[0]), torch.empty_like(rel[1])
    ws = torch.empty(B.ssam_sparse_attention_backward_workspace_bytes(groups, S, w, h, d), dtype=torch.uint8, device=DEV)
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    places = lambda t: [C.c_void_p(t.data_ptr() + 2 * x) for x in at]  # noqa: E731
    rc = B.lib().ssam_sparse_attention_backward(*places(src), C.c_long(row), p(rel[0]), p(rel[1]), p(sigma), C.c_long(S), p(out), p(dout), None, *places(dst), C.c_long(row), p(dh), p(dw),
                                                groups, S, w, h, d, tile, C.c_double(0.5), C.c_float(d ** -0.5), p(ws), C.c_size_t(ws.numel()),
                                                C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    torch.cuda.synchronize()
    for i in range(3):
        assert torch.equal(dst[:, at[i]:at[i] + h * d], want[:, :, i].reshape(groups * S, h * d))
        if i < 2:
            assert bool(dst[:, at[i] + h * d:at[i] + h * d + 4096].isnan().all())
    assert torch.equal(dh, wh) and torch.equal(dw, ww)


def test_many_windows():
    """8912896 (group, head) of one token, more than a grid's limit of 8388600: P is 1 and dS is dO.(v - out), 0 where out is v, so dV is dO and the rest is 0."""
    announce("sparse_attention_backward many windows")
    groups, h, d = 1 << 19, 17, 16
    g = T.gen(1)
    qkv = torch.randn(groups, 1, 3, h, d, generator=g, device=DEV, dtype=torch.float32).to(BF)
    rel = [T.normal(g, 1, d, std=0.1, dtype=BF) for _ in range(2)]
    sigma = torch.zeros(1, dtype=torch.int32, device=DEV)
    dout = torch.randn(groups, h * d, generator=g, device=DEV, dtype=torch.float32).to(BF)
    out = qkv[:, 0, 2].reshape(groups, h * d).contiguous()
    dqkv, drel_h, drel_w = B.ssam_sparse_attention_backward(qkv, *rel, sigma, 1, 32, 1.0, out, dout)
    assert torch.equal(dqkv[:, 0, 2].reshape(groups, h * d), dout)
    # dP is a product of 16 terms in matrix instructions, delta the same by one lane after the other: 16 additions in 32 bits off by 2^-24 of a sum below 16 * 6 * 6
    assert float(dqkv[:, 0, :2].float().abs().max()) <= 16 * 2.0 ** -24 * 576 * 6 * 2
    assert bool(torch.isfinite(drel_h).all()) and bool(torch.isfinite(drel_w).all())


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
