"""Gradients of attention by norms against 64-bit formulas (attention_gradient_reference, which derives the bounds): every kernel that a call can choose, many (group, head), the tables'
share by itself, scores that climb along the scan so that the running sums are rescaled again and again, and differences of the forward's value."""
import math

import pytest
import torch

import attention_gradient_reference as R
import test_gpu_attention_gradients as T
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16

# (groups, side, heads, head size, mask tile, density, order, dropped queries)
GRIDS = [
    # sides up to 16: every head size, orders of all groups and of one, more than eight (group, head) and no multiple of eight
    (1, 15, 3, 64, 128, 0.5, "content", True), (2, 15, 2, 80, 128, 0.5, "position", False), (1, 15, 9, 16, 128, 1.0, "content", False), (1, 16, 9, 32, 128, 0.5, "position", False),
    (2, 16, 3, 80, 128, 0.5, "content", True),
    # up to 32: small heads; 32 is a power of two (stages of slices, of 80 features with dO in LDS), the others are not
    (1, 17, 2, 16, 128, 0.4, "position", False), (1, 31, 2, 32, 128, 0.4, "content", True), (2, 32, 5, 16, 128, 0.5, "position", False), (1, 32, 3, 32, 128, 0.5, "position", True),
    (1, 32, 2, 32, 128, 0.6, "content", False), (1, 32, 2, 80, 128, 0.4, "position", True), (3, 28, 4, 64, 128, 0.5, "content", True), (1, 30, 11, 80, 128, 0.3, "position", False),
    # the prefix's keys in one slice of the queries, stored without a join: more than 256 tiles
    (9, 32, 8, 64, 128, 0.5, "position", False), (1, 64, 24, 64, 128, 0.4, "position", False), (3, 64, 8, 80, 128, 0.4, "position", False),
    # up to 64
    (2, 64, 8, 80, 128, 0.4, "position", False), (1, 64, 3, 32, 128, 0.3, "position", True), (1, 64, 9, 16, 128, 0.2, "position", False), (2, 50, 5, 64, 128, 0.4, "content", False),
    (1, 33, 9, 80, 128, 0.5, "position", False), (1, 64, 2, 80, 128, 1.0, "content", False),
    # above: 128 x 128 in the position-only order, the only call of its kernel, and others
    (1, 128, 2, 64, 128, 0.1, "position", False), (1, 128, 1, 80, 128, 0.1, "position", True), (1, 128, 1, 16, 128, 0.05, "position", False), (1, 128, 1, 32, 128, 0.3, "position", False),
    (3, 66, 3, 80, 128, 0.3, "content", True), (1, 100, 9, 64, 128, 0.2, "position", False), (2, 72, 1, 16, 128, 0.0001, "content", False), (1, 127, 2, 32, 128, 0.1, "position", False),
]
WINDOWS = [(2, 14, 5, 80, 32, 0.5, "content", True), (30, 14, 12, 64, 32, 0.4, "position", False), (5, 14, 3, 16, 32, 1.0, "content", False), (2, 14, 9, 32, 32, 0.0001, "position", False),
           (3, 13, 3, 80, 128, 0.5, "content", False), (40, 8, 12, 64, 32, 0.5, "position", True), (9, 7, 3, 80, 32, 0.5, "content", False)]


def call(inputs, case, scale=None):
    qkv, rel, sigma, out_rows, dout, rows = inputs
    groups, w, h, d, tile, r = case[:6]
    out = torch.zeros(rows, h * d, dtype=BF, device=DEV)
    B.ssam_sparse_attention(qkv, *rel, sigma, w, tile, r, out=out, out_rows=out_rows)
    return out, B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, dout, out_rows=out_rows)


def against(inputs, case, out, got, **kw):
    qkv, rel, sigma, out_rows, dout, _ = inputs
    R.check(got, *R.gradients(qkv, rel, sigma, case[1], case[4], case[5], dout, out, out_rows), str(case), **kw)


@pytest.mark.parametrize("case", GRIDS + WINDOWS)
def test_norms(case):
    announce("sparse_attention_backward norms", case)
    inputs = T.inputs(case[1] + case[2], *case[:4], case[6], case[7])
    out, got = call(inputs, case)
    against(inputs, case, out, got)


@pytest.mark.parametrize("case", [(2, 14, 2, 64, 32, 0.5, "content", False), (1, 14, 3, 80, 32, 0.4, "position", True), (1, 28, 2, 64, 128, 0.5, "position", False), (1, 32, 2, 80, 128, 0.4, "position", False),
                                  (1, 24, 2, 32, 128, 0.5, "content", True), (1, 64, 2, 64, 128, 0.4, "position", False), (1, 50, 2, 80, 128, 0.4, "content", False)])
def test_through_the_tables(case):
    """Small queries and large tables: dQ and the tables' gradients are what comes through G.  On grids up to 32 x 32 and in windows G takes dS as the sum of two bf16 and is multiplied as two, so
    that nothing but the result's rounding is left (1.07 of it; half a bias of 0.4 in fp16 and G in fp16 add 2e-4 in the squares); above, the rounding of dS, which the reference counts."""
    announce("sparse_attention_backward through the tables", case)
    qkv, rel, sigma, out_rows, dout, rows = T.inputs(case[1], *case[:4], case[6], case[7], rel_std=1.0)
    qkv[:, :, 0] = (qkv[:, :, 0].float() * (0.05 / 0.7)).to(BF)
    inputs = (qkv, rel, sigma, out_rows, dout, rows)
    out, got = call(inputs, case)
    groups, w, h, d, tile, r = case[:6]
    single, table = R.gradients(qkv, rel, sigma, w, tile, r, dout, out, out_rows)
    for (g, x), (grads, loss) in single.items():
        R.off(got[0][g, :, 0, x], grads[0], loss[0], f"dq {case}", factor=1.07, small=1.5e-4)
    for i, name in enumerate(("drel_h", "drel_w")):
        R.off(got[1 + i], table[0][i], table[1][i], f"{name} {case}", factor=1.07, small=1.5e-4)


# of 64 x 64 in the position-only order the row walk has a rescaling of its own (eight slices of G), of 80 features with other stages
CLIMBS = [(2, 14, 2, 64, 32, 1.0, "position", False), (1, 14, 3, 80, 32, 1.0, "content", True), (1, 28, 2, 64, 128, 0.6, "content", False), (1, 32, 2, 64, 128, 0.6, "position", False),
          (1, 32, 2, 80, 128, 1.0, "position", False), (1, 64, 2, 64, 128, 0.4, "position", False), (1, 64, 2, 80, 128, 0.4, "position", True), (1, 64, 1, 16, 128, 0.4, "position", False),
          (1, 50, 1, 80, 128, 0.4, "content", False), (1, 72, 2, 64, 128, 0.4, "content", False), (1, 128, 1, 64, 128, 0.1, "position", False)]


@pytest.mark.parametrize("case", CLIMBS)
def test_climbing_scores(case):
    """Queries share a direction along which the keys grow with their place in the scan: within the prefix the largest score of a query rises by 2^50 (in windows by 2^84), in steps that move the
    reference of its running sums three times and more for most queries, which is counted.  Few keys have all the weight, of a window's queries three to five, so that
    fewer roundings make up a norm: 1.5 of it there."""
    announce("sparse_attention_backward climbing scores", case)
    groups, w, h, d, tile, r, order, drop = case
    qkv, rel, sigma, out_rows, dout, rows = T.inputs(8, groups, w, h, d, order, drop, rel_std=0.01)
    S = w * w
    u = (torch.randint(0, 2, (d,), generator=T.gen(9), device=DEV) * 2 - 1) * d ** -0.5
    climb = (84 if w <= 14 else 50) / (R.prefix(S, tile, r) * tile / S)
    rise = climb / (40 * d ** -0.5 * math.log2(math.e))
    x = qkv.float()
    x[:, :, 0] += 40 * u
    x[:, :, 1] -= (x[:, :, 1] @ u)[..., None] * u                         # (what keys have of it by chance would be a noise of several units)
    x[:, :, 1] += torch.linspace(0, rise, S, device=DEV)[None, :, None, None] * u
    inputs = (x.to(BF), rel, sigma, out_rows, dout, rows)
    q, k = (inputs[0][0, :, i, 0].double() for i in range(2))
    L, _ = R.scores(q, k, *[t.double() for t in rel], (sigma[0] if sigma.dim() == 2 else sigma).long(), w, tile, r, d ** -0.5, torch.arange(0, S, max(1, S // 512), device=DEV))
    assert float((R.moves(L) >= 3).double().mean()) > 0.5
    out, got = call(inputs, case)
    against(inputs, case, out, got, factor=1.5 if w <= 14 else 1.25, small=6e-4)


@pytest.mark.parametrize("case", [(1, 7, 1, 32, 32, 0.5, "content", False), (1, 14, 1, 80, 32, 0.5, "position", False), (1, 17, 1, 64, 128, 0.4, "content", False), (1, 32, 1, 16, 128, 0.5, "position", False)])
def test_differences(case):
    """The slope of sum(result * dout) in 64 bits, by central differences, along the gradient itself and along random directions.  The kernels' error has a norm E at most: their roundings
    (as in test_norms) and what delta loses with the forward's rounded result, which is worked out.  Along the gradient the slope is off by E at most, along a random direction by E
    times a normal deviate, 6 at most: a gradient of zeros, or one that is 2 % too large, fails."""
    announce("sparse_attention_backward differences", case)
    groups, w, h, d, tile, r, order, drop = case
    inputs = T.inputs(12, *case[:4], order, drop)
    qkv, rel, sigma, _, dout, _ = inputs
    out, (dqkv, *drel) = call(inputs, case)
    s = (sigma[0] if sigma.dim() == 2 else sigma).long()
    leaves = [qkv[0, :, i, 0].double() for i in range(3)] + [t.double() for t in rel]
    mine = [dqkv[0, :, i, 0].double() for i in range(3)] + [t.double() for t in drel]
    do, scale, at = dout.double().view(-1, d), d ** -0.5, torch.arange(w * w, device=DEV)

    def result(leaves):
        return torch.softmax(R.scores(leaves[0], leaves[1], leaves[3], leaves[4], s, w, tile, r, scale, at)[0], 1) @ leaves[2]

    head = (s, w, tile, r, do)
    true, loss = R.one_head(*leaves, *head, result(leaves), scale, w <= 32)
    near, _ = R.one_head(*leaves, *head, out.double().view(-1, d), scale, w <= 32)
    g = T.gen(13)
    for leaf in range(5):
        E = 1.2 * math.sqrt(float(R.lost(true[leaf]).sum() + loss[leaf].sum())) + 4e-4 * float(true[leaf].norm()) + float((near[leaf] - true[leaf]).norm())
        assert E <= 0.02 * float(true[leaf].norm())
        for turn in range(5):
            u = torch.randn(leaves[leaf].shape, generator=g, device=DEV, dtype=torch.float64) if turn else true[leaf] / true[leaf].norm()
            # a step that moves scores by a few 1e-5 at most: differences are off by its square, and by 2^-53 over it
            step = 1e-4 / max(1.0, float(u.abs().max()))
            ends = [float((result([t + sign * step * u if i == leaf else t for i, t in enumerate(leaves)]) * do).sum()) for sign in (1, -1)]
            slope, got = (ends[0] - ends[1]) / (2 * step), float((mine[leaf] * u).sum())
            assert abs(got - slope) <= (6 if turn else 1) * E + 1e-6 * float((true[leaf] * u).abs().sum()), (leaf, turn, got, slope, E)
