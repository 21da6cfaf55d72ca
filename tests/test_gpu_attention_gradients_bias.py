"""Gradients of attention in windows with biases past 65504 times the scale, which the forward call holds, against 64 bits; and scales at both ends of what the call takes."""
import pytest
import torch

import attention_gradient_reference as R
import test_gpu_attention_gradients as T
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16


@pytest.mark.parametrize("d", [16, 64, 80])
@pytest.mark.parametrize("scale,low,high", [(0.125, 8320.0, 8960.0), (2.0 ** -9, 200.0, 400.0), (2.0 ** -9, -400.0, -200.0), (2.0 ** -6, 2048.0, 4096.0)])
def test_biases_past_fp16(scale, low, high, d):
    """Keys three rows above a query and further have a bias of `low`, from six rows on of `high`: where both were held at the same bound, the first would keep their weight.
    Scores of 9000 in 32 bits are off by 2^-11 a sum at most, 3e-4 of a probability at the root of the mean square and 8e-4 after d / 16 + 2 of them: `factor` and `small` make room for it.
    dQ's first feature is a sum of G over keys whose G cancels, times thousands: it is left out."""
    announce("sparse_attention_backward biases past fp16", scale, low, high, d)
    w, groups, h = 14, 2, 2
    qkv, rel, sigma, _, dout, rows = T.inputs(d, groups, w, h, d, "content", False)
    qkv[:, :, 0, :, 0] = 4.0
    for t, bias in ((slice(w + 2, w + 5), low), (slice(w + 5, None), high)):
        rel[0][t] = 0.0
        rel[0][t, 0] = bias / 4
        assert (rel[0][t, 0].double() * 4 == bias).all()
    out = torch.zeros(rows, h * d, dtype=BF, device=DEV)
    B.ssam_sparse_attention(qkv, *rel, sigma, w, 32, 0.5, scale=scale, out=out)
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, 32, 0.5, out, dout, scale=scale)
    single, table = R.gradients(qkv, rel, sigma, w, 32, 0.5, dout, out, scale=scale)
    for grads, loss in single.values():
        grads[0][:, 0] = loss[0][:, 0] = 0.0
    assert torch.isfinite(got[0]).all()
    got[0][:, :, 0, :, 0] = 0.0
    R.check(got, single, table, f"scale {scale} biases {low} {high} d={d}", factor=1.3, small=1e-3)


@pytest.mark.parametrize("w,tile,order", [(14, 32, "content"), (14, 128, "position"), (16, 128, "content"), (32, 128, "position")])
@pytest.mark.parametrize("scale", [2.0 ** -9, 0.02, 0.7, 1.0, 300.0, 512.0])
def test_scales(scale, w, tile, order):
    """Queries and tables of the sizes that give logits and biases of a few units at this scale: logits have a deviation of 1, biases of 0.5."""
    announce("sparse_attention_backward scales", scale, w, tile, order)
    groups, h, d = 1, 2, 64
    qkv, rel, sigma, _, dout, rows = T.inputs(3, groups, w, h, d, order, False)
    size = 1 / (scale * 0.7 * d ** 0.5)
    qkv[:, :, 0] *= size / 0.7
    rel = [(t * (0.5 / (0.1 * size * d ** 0.5))).to(BF) for t in rel]
    out = torch.zeros(rows, h * d, dtype=BF, device=DEV)
    B.ssam_sparse_attention(qkv, *rel, sigma, w, tile, 0.5, scale=scale, out=out)
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, 0.5, out, dout, scale=scale)
    R.check(got, *R.gradients(qkv, rel, sigma, w, tile, 0.5, dout, out, scale=scale), f"scale {scale} {w} {tile}")
