"""The formulas that the GPU's gradients are held against (attention_gradient_reference), on the CPU: against automatic differentiation, against differences, and that
their bounds see a mistake, which is put into the formulas' own result."""
import math

import pytest
import torch

import attention_gradient_reference as R

CASES = [(1, 16, 32, 1.0), (4, 16, 32, 0.5), (7, 16, 32, 0.5), (14, 32, 32, 0.3), (17, 16, 128, 0.4)]


def inputs(w, d, seed=0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: torch.randn(*s, generator=g, dtype=torch.float64) * std  # noqa: E731
    S = w * w
    return [n(S, d, std=0.7), n(S, d, std=0.7), n(S, d, std=0.7), n(2 * w - 1, d, std=0.3), n(2 * w - 1, d, std=0.3)], torch.randperm(S, generator=g), n(S, d)


def result(leaves, sigma, w, tile, r, scale):
    L, _ = R.scores(leaves[0], leaves[1], leaves[3], leaves[4], sigma, w, tile, r, scale, torch.arange(w * w))
    return torch.softmax(L, 1) @ leaves[2]


@pytest.mark.parametrize("w,d,tile,r", CASES)
def test_formulas(w, d, tile, r):
    leaves, sigma, do = inputs(w, d)
    scale = d ** -0.5
    at = [t.clone().requires_grad_() for t in leaves]
    out = result(at, sigma, w, tile, r, scale)
    out.backward(do)
    grads, _ = R.one_head(*leaves, sigma, w, tile, r, do, out.detach(), scale, True)
    for got, leaf in zip(grads, at):
        assert float((got - leaf.grad).abs().max()) <= 1e-12 * (1 + float(leaf.grad.abs().max()))
    g = torch.Generator().manual_seed(1)
    for i in range(5):
        u = torch.randn(leaves[i].shape, generator=g, dtype=torch.float64)
        ends = [float((result([t + s * 1e-5 * u if j == i else t for j, t in enumerate(leaves)], sigma, w, tile, r, scale) * do).sum()) for s in (1, -1)]
        # a central difference of 1e-5 is off by 1e-10 of third derivatives of a few units a term, and by 2^-53 / 1e-5 of the terms
        assert abs((ends[0] - ends[1]) / 2e-5 - float((grads[i] * u).sum())) <= 1e-7 * (1 + float((grads[i] * u).abs().sum()))


def test_bounds_see_what_they_are_for():
    """Results rounded as the kernels round them pass; a factor of 1 %, a missing term and G from dS as one bf16 do not."""
    w, d, tile, r = 14, 32, 32, 0.5
    leaves, sigma, do = inputs(w, d, 3)
    scale = d ** -0.5
    out = result(leaves, sigma, w, tile, r, scale)
    grads, loss = R.one_head(*leaves, sigma, w, tile, r, do, out, scale, True)
    L, back = R.scores(leaves[0], leaves[1], leaves[3], leaves[4], sigma, w, tile, r, scale, torch.arange(w * w))
    p = torch.softmax(L, 1)
    ds = p * (do @ leaves[2].T - (do * out).sum(1, keepdim=True))
    b = lambda t: t.to(R.BF).double()  # noqa: E731
    G = lambda m: torch.zeros(w * w, 2 * w - 1, dtype=torch.float64).scatter_add_(1, back[0], m)  # noqa: E731
    R.off(b(b(p).T @ do), grads[2], loss[2], "dv")
    R.off(b(b(ds).T @ leaves[0] * scale), grads[1], loss[1], "dk")
    R.off(b(G(ds).T @ leaves[0]), grads[3], loss[3], "drel_h", factor=1.07, small=1.5e-4)
    for bad, i in ((1.01 * grads[2], 2), (grads[1] * 0.99, 1), (grads[0] - G(ds) @ leaves[3], 0)):
        with pytest.raises(AssertionError):
            R.off(bad, grads[i], loss[i], "planted")
    with pytest.raises(AssertionError):
        R.off(b(G(b(ds)).T @ leaves[0]), grads[3], loss[3], "drel_h from one bf16", factor=1.07, small=1.5e-4)


def test_climbing_scores_are_counted():
    """moves() of the GPU's tests, on a case that can be counted by hand."""
    L = torch.tensor([[0.0, 10.0, 12.0, 30.0], [5.0, 4.0, 3.0, 2.0]], dtype=torch.float64).repeat_interleave(32, 1) / math.log2(math.e)
    assert R.moves(L).tolist() == [2, 0]
