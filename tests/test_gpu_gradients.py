"""Gradient of the gathered LayerNorm, and activations in 8 bits with the GELU that reads them, against plain 64-bit arithmetic.

Tolerances: a bf16 result is off by at most half a step, 2^-8 of the value, and what 32-bit sums add to it; each test says how much."""
import math

import numpy as np
import pytest
import torch

from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
EPS = 1e-6
HALF = 2.0 ** -8


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def close(got, ref, slack, what):
    """Every element within half a step of bf16 of the reference, and `slack` more."""
    got, ref = got.double(), ref.double()
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() - HALF * ref.abs() - slack
    assert (over <= 0).all(), f"{what}: {float(over.max()):.3e} past the bound at {int(over.argmax())}"


# ------------------------------------------------------------------ LayerNorm
def ln_reference(x, idx, gamma, dy, dx0, accumulate):
    """-> dx, dgamma, dbeta in 64 bits; how far 32-bit arithmetic may be off dx; sums of magnitudes for the weights' gradients"""
    x, gamma, dy, dx = x.double(), gamma.double(), dy.double(), dx0.double().clone()
    D = x.shape[2]
    slack = torch.zeros_like(dx)
    dgamma, dbeta, m_gamma, m_beta = (torch.zeros(D, dtype=torch.float64, device=DEV) for _ in range(4))
    for b in range(x.shape[0]):
        i = idx[b % idx.shape[0]].long()
        p = torch.nonzero((i >= 0) & (i < x.shape[1]))[:, 0]
        rows = x[b, i[p]]
        dev = rows - rows.mean(1, keepdim=True)
        rstd = ((dev ** 2).mean(1, keepdim=True) + EPS).rsqrt()
        h, d = dev * rstd, dy[b, p]
        g = d * gamma
        out = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        dx[b, i[p]] = out + (dx[b, i[p]] if accumulate else 0)
        # sums of at most 2048 terms are off by under 40 * 2^-24 of their magnitudes (32 terms a lane, six exchanges); rows are centred about
        # a mean off by that much of their largest value
        off = 2.0 ** -18 * (1 + rows.abs().amax(1, keepdim=True) * rstd)
        slack[b, i[p]] = off * rstd * g.abs().amax(1, keepdim=True) * (2 + h.abs()) * 2
        dgamma += (d * h).sum(0)
        dbeta += d.sum(0)
        m_gamma += (d * h).abs().sum(0) + off.max() * d.abs().sum(0) * 2 ** 6
        m_beta += d.abs().sum(0)
    return dx, dgamma, dbeta, slack, m_gamma, m_beta


# (images, tokens, output rows, features, table per image, added)
LN_CASES = [(1, 1, 1, 8, False, False), (2, 7, 5, 24, True, True), (1, 3, 64, 520, False, False), (3, 50, 70, 1032, True, True), (2, 64, 64, 512, False, True),
            (2, 100, 90, 768, True, False), (2, 300, 313, 1280, False, True), (1, 40, 37, 1536, True, True), (2, 33, 21, 2048, True, False), (2, 33, 40, 2048, False, True),
            (1, 5000, 4900, 144, True, True), (2, 4096, 4900, 1024, False, True)]


def ln_inputs(Bn, N, Nout, D, own_table, seed):
    g = gen(seed)
    tables = Bn if own_table else 1
    idx = torch.full((tables, Nout), -1, dtype=torch.int32, device=DEV)
    for t in range(tables):                                 # no row twice; what the rows do not fill is a padding slot, at any place
        k = min(N, Nout) - (1 if min(N, Nout) > 2 else 0)
        at = torch.randperm(Nout, generator=g, device=DEV)[:k]
        idx[t, at] = torch.randperm(N, generator=g, device=DEV)[:k].to(torch.int32)
    if Nout > 3:
        idx[0, (idx[0] < 0).nonzero()[:1, 0]] = N           # past the rows: none, as a negative one
    x = normal(g, Bn, N, D, dtype=BF) * torch.exp(normal(g, Bn, N, 1)).to(BF) + normal(g, 1, 1, D, std=0.5, dtype=BF)
    return x, idx, 1 + normal(g, D, std=0.2), normal(g, Bn, Nout, D, std=0.02, dtype=BF), normal(g, Bn, N, D, std=0.02, dtype=BF)


@pytest.mark.parametrize("case", LN_CASES)
def test_layernorm_gradient(case):
    announce("ln_gather_backward", case)
    Bn, N, Nout, D, own_table, accumulate = case
    x, idx, gamma, dy, dx0 = ln_inputs(Bn, N, Nout, D, own_table, sum(case))
    stride = Nout if own_table else 0
    dx, dgamma, dbeta = B.ssam_ln_gather_backward(x, idx, stride, gamma, EPS, dy, dx=dx0.clone(), accumulate=accumulate)
    ref, rg, rb, slack, mg, mb = ln_reference(x, idx, gamma, dy, dx0, accumulate)
    close(dx, ref, slack, "dx")
    untouched = slack.amax(2) == 0
    assert torch.equal(dx[untouched], dx0[untouched]), "a row that idx does not name changed"
    # at most 16 rows a wave here, four waves, 16 + 5 sums of workgroups: under 64 additions of 2^-24, and the error of h
    for got, want, size, what in ((dgamma, rg, mg, "dgamma"), (dbeta, rb, mb, "dbeta")):
        assert ((got.double() - want).abs() <= 2.0 ** -18 * size + 1e-30).all(), what
    again = B.ssam_ln_gather_backward(x, idx, stride, gamma, EPS, dy, dx=dx0.clone(), accumulate=accumulate)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma) and torch.equal(again[2], dbeta), "another result for the same inputs"
    only, none, _ = B.ssam_ln_gather_backward(x, idx, stride, gamma, EPS, dy, dx=dx0.clone(), accumulate=accumulate, weight_grads=False)
    assert torch.equal(only, dx) and none is None


def test_layernorm_gradient_of_the_forward_call():
    """Against differences of ssam_ln_gather's own definition in 64 bits, along a direction in x, gamma and beta."""
    announce("ln_gather_backward against differences")
    Bn, N, Nout, D = 2, 20, 24, 136
    x, idx, gamma, dy, _ = ln_inputs(Bn, N, Nout, D, True, 5)
    beta = normal(gen(6), D)
    y = B.ssam_ln_gather(x, idx, Nout, gamma, beta, EPS, Nout)

    def forward(x, gamma, beta):
        out = torch.zeros(Bn, Nout, D, dtype=torch.float64, device=DEV)
        for b in range(Bn):
            p = torch.nonzero((idx[b] >= 0) & (idx[b] < N))[:, 0]
            out[b, p] = torch.nn.functional.layer_norm(x[b, idx[b, p].long()], (D,), gamma, beta, EPS)
        return out

    at = [t.double() for t in (x, gamma, beta)]
    close(y, forward(*at), 1e-5 * float(y.abs().max()), "forward")
    dx, dgamma, dbeta = B.ssam_ln_gather_backward(x, idx, Nout, gamma, EPS, dy)
    for k, grad in enumerate((dx, dgamma, dbeta)):
        way = torch.randn(at[k].shape, generator=gen(k), device=DEV, dtype=torch.float64)
        step = 1e-5
        ends = [sum((forward(*[t + s * step * way if j == k else t for j, t in enumerate(at)]) * dy.double()).flatten().tolist()) for s in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * step)
        # every element of the gradient is off by at most 2^-8 of itself; the differences' own error is far below
        assert abs(slope - float((grad.double() * way).sum())) <= HALF * float((grad.double() * way).abs().sum()) + 1e-6, k


def test_layernorm_gradient_without_rows():
    announce("ln_gather_backward: no row named")
    x, idx, gamma, dy, dx0 = ln_inputs(2, 9, 12, 64, False, 1)
    idx.fill_(-1)
    dx, dgamma, dbeta = B.ssam_ln_gather_backward(x, idx, 0, gamma, EPS, dy * float("nan"), dx=dx0.clone(), accumulate=True)
    assert torch.equal(dx, dx0) and not dgamma.any() and not dbeta.any()
    dx, _, _ = B.ssam_ln_gather_backward(x, idx, 0, gamma, EPS, dy)
    assert not dx.any()


def test_layernorm_gradient_does_not_spread_what_is_not_finite():
    announce("ln_gather_backward: NaN in padding rows and in rows that are not named")
    x, idx, gamma, dy, dx0 = ln_inputs(1, 30, 40, 264, False, 2)
    want = B.ssam_ln_gather_backward(x, idx, 0, gamma, EPS, dy, dx=dx0.clone(), accumulate=True)
    pad = (idx[0] < 0) | (idx[0] >= 30)
    dy[0, pad] = float("nan")
    left = torch.ones(30, dtype=torch.bool, device=DEV)
    left[idx[0][~pad].long()] = False
    x[0, left] = float("inf")
    got = B.ssam_ln_gather_backward(x, idx, 0, gamma, EPS, dy, dx=dx0.clone(), accumulate=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------ 8 bits
def held(x):
    """-> codes * 1 and scale per column in 64 bits, and where the code is no tie within 32-bit rounding"""
    rows, D = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -D % 64)).view(rows, -1, 64)
    top = v.abs().amax(2, keepdim=True)
    scale = (top / 127).clamp(min=2.0 ** -126)
    exact = torch.where(top > 0, v / scale, 0.0)
    sure = ((exact - exact.floor() - 0.5).abs() > 2.0 ** -15)            # 127 * 2^-23 twice: the factor's rounding and the product's
    code = exact.round()
    cut = lambda t: t.expand_as(v).flatten(1)[:, :D]  # noqa: E731
    return cut(code), cut(scale), cut(sure)


SHAPES = [(1, 8), (1, 64), (3, 72), (5, 56), (7, 144), (33, 576), (2, 1000), (513, 768), (4, 5120), (9, 10248)]


@pytest.mark.parametrize("rows,D", SHAPES)
def test_checkpoint(rows, D):
    announce("checkpoint", rows, D)
    g = gen(rows + D)
    x = (normal(g, rows, D) * torch.exp(2 * normal(g, rows, D))).to(BF)
    codes, scales = B.ssam_checkpoint_store(x)
    code, scale, sure = held(x)
    assert codes.dtype == torch.int8 and codes.shape == x.shape and scales.shape == (rows, -(-D // 64))
    off = (codes.double() - code).abs()
    assert (off[sure] == 0).all() and (off <= 1).all()
    per_column = scales.repeat_interleave(64, 1)[:, :D].double()
    assert ((per_column - scale).abs() <= 2.0 ** -23 * scale).all()
    back = B.ssam_checkpoint_restore(codes, scales)
    close(back, codes.double() * per_column, 2.0 ** -23 * scale * 127, "restored")        # the product is rounded to 32 bits, then to bf16
    top = scale * 127
    assert ((back.double() - x.double()).abs() <= top / 254 * (1 + 2.0 ** -12) + HALF * back.double().abs()).all()
    assert torch.equal(B.ssam_checkpoint_restore(codes, scales, x=torch.empty_like(x)), back)


def test_checkpoint_of_what_is_not_ordinary():
    announce("checkpoint: zeros, infinities, NaN, the smallest and the largest values")
    x = torch.zeros(8, 136, dtype=BF, device=DEV)
    x[1, 3], x[2, 70], x[3, 135] = float("inf"), float("nan"), float("-inf")
    x[4, :64] = torch.finfo(BF).max
    x[4, 1] = -torch.finfo(BF).max
    x[5, :64], x[5, 64] = torch.finfo(BF).tiny, -2.0 ** -133
    x[6], x[6, 5] = 1.0, -1.0
    x[7, 0] = -0.0
    codes, scales = B.ssam_checkpoint_store(x)
    back = B.ssam_checkpoint_restore(codes, scales)
    for row, block in ((1, 0), (2, 1), (3, 2)):                          # that block and no other
        at = slice(64 * block, min(64 * block + 64, 136))
        assert back[row, at].isnan().all() and int(back[row].isnan().sum()) == at.stop - at.start
        assert not codes[row].any()
    assert not back[0].any() and not back[7].any()
    assert torch.equal(back[4], x[4]) and torch.equal(back[6], x[6])     # 127 times 1/127 of a power of two, or of the largest, rounds back
    assert ((back[5].double() - x[5].double()).abs() <= 2.0 ** -127).all()


@pytest.mark.parametrize("rows,D", SHAPES)
def test_gelu_through_8_bits(rows, D):
    announce("gelu", rows, D)
    g = gen(rows * 3 + D)
    h, da = (normal(g, rows, D, std=2.0) * torch.exp(normal(g, 1, D))).to(BF), normal(g, rows, D, std=0.02, dtype=BF)
    a, codes, scales = B.ssam_gelu_checkpoint(h)
    want = B.ssam_checkpoint_store(h)
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    phi = lambda t: 0.5 * torch.erfc(-t * math.sqrt(0.5))  # noqa: E731
    # the approximation of erfc is off by 1.5e-7 at most, half of it counts, and 32-bit arithmetic about as much: 3e-7 |t| and 3e-7
    close(a, h.double() * phi(h.double()), 3e-7 * h.double().abs(), "a")
    t = codes.double() * scales.repeat_interleave(64, 1)[:, :D].double()
    dh, again = B.ssam_gelu_backward(codes, scales, da)
    close(again, t * phi(t), 4e-7 * t.abs(), "a again")
    slope = phi(t) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)
    close(dh, da.double() * slope, 6e-7 * da.double().abs(), "dh")
    # in place, and without the activation
    own = h.clone()
    B.ssam_gelu_checkpoint(own, a=own)
    assert torch.equal(own, a)
    grad = da.clone()
    assert B.ssam_gelu_backward(codes, scales, grad, dh=grad, activation=False) == (grad, None)
    assert torch.equal(grad, dh)


def test_gelu_gradient_against_differences():
    announce("gelu against differences")
    h = torch.linspace(-9, 9, 64 * 9, device=DEV).view(9, 64).to(BF)
    _, codes, scales = B.ssam_gelu_checkpoint(h)
    dh, _ = B.ssam_gelu_backward(codes, scales, torch.ones_like(h))
    t = codes.double() * scales.double()
    f = lambda t: t * 0.5 * torch.erfc(-t * math.sqrt(0.5))  # noqa: E731
    close(dh, (f(t + 1e-4) - f(t - 1e-4)) / 2e-4, 1e-6, "dh")


def test_gradients_on_another_stream_and_in_a_graph():
    """Calls on a stream of the caller's, and captured, replayed three times with eager work between."""
    announce("gradients: stream and graph")
    x, idx, gamma, dy, dx0 = ln_inputs(2, 300, 313, 768, True, 9)
    h, da = normal(gen(3), 626, 1024, dtype=BF), normal(gen(4), 626, 1024, std=0.02, dtype=BF)
    dx, a, dh = dx0.clone(), torch.empty_like(h), torch.empty_like(h)
    codes, scales = torch.empty(h.shape, dtype=torch.int8, device=DEV), torch.empty(626, 16, device=DEV)
    ws = torch.empty(B.ssam_ln_gather_backward_workspace_bytes(2, 313, 768), dtype=torch.uint8, device=DEV)

    def step():
        dx.copy_(dx0)
        _, dg, db = B.ssam_ln_gather_backward(x, idx, 313, gamma, EPS, dy, dx=dx, accumulate=True, workspace=ws)
        B.ssam_gelu_checkpoint(h, a=a, codes=codes, scales=scales)
        B.ssam_gelu_backward(codes, scales, da, dh=dh, a=a)
        return dx, dg, db, dh, a

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        got = step()
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want)), turn
        B.ssam_gelu_backward(*B.ssam_checkpoint_store(h), da)
        torch.cuda.synchronize()
