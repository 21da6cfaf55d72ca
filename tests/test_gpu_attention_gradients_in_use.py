"""Gradients of Stripe-Sort attention where a call can go wrong: differences of the forward's value, many (group, head) to a workgroup, orders that are not the product's,
scores that grow along the keys, what lies in rows that no gradient comes from, rows of any stride, streams and graphs; and the gradient calls of a block together.

Bounds of single gradients are those of test_gpu_attention_gradients (its docstring derives them)."""
import ctypes as C
import math

import pytest
import torch

import test_gpu_attention_gradients as T
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16


def against_64_bits(case, inputs, got, scale=None):
    groups, w, h, d, tile, r, order, drop = case
    qkv, rel, sigma, out_rows, dout, out = inputs
    grads, size, drel, drel_size = T.reference(qkv, *rel, sigma, w, tile, r, dout, out_rows, scale or d ** -0.5)
    for i, name in enumerate("qkv"):
        T.check(got[0][:, :, i], grads[:, :, i], size[:, :, i], f"d{name} {case}")
    for name, a, b, s in zip(("drel_h", "drel_w"), got[1:], drel, drel_size):
        T.check(a, b, s, name)


# one tile and more of the dense prefix of a window, all of them, and none; both mask tiles; more (group, head) than there are CUs, and not a multiple of eight
WINDOWS = [(1, 14, 2, 64, 32, 0.05, "position", False), (2, 14, 1, 80, 32, 0.15, "content", False), (1, 14, 3, 32, 32, 0.3, "position", True), (2, 14, 1, 16, 32, 0.45, "content", False),
           (1, 14, 2, 80, 32, 0.6, "content", True), (1, 14, 1, 64, 32, 0.75, "position", False), (1, 14, 1, 80, 32, 0.9, "position", False), (1, 14, 2, 80, 32, 1.0, "content", False),
           (1, 14, 2, 80, 128, 0.4, "content", False), (1, 14, 2, 64, 128, 0.5, "position", True), (1, 14, 1, 32, 128, 1.0, "position", False), (3, 7, 2, 64, 32, 0.5, "content", True),
           (1, 3, 5, 80, 128, 1.0, "position", False), (23, 7, 12, 16, 32, 0.5, "content", True), (19, 14, 16, 80, 32, 0.4, "position", False)]


@pytest.mark.parametrize("case", WINDOWS)
def test_windows(case):
    announce("sparse_attention_backward windows", case)
    inputs, got = T.run(case, seed=case[0] + case[1])
    against_64_bits(case, inputs, got)


@pytest.mark.parametrize("w,d", [(16, 64), (32, 64), (64, 32)])
def test_an_order_of_all_groups_that_scatters(w, d):
    """Shared by the groups, on a grid of a power of two, but not the product's order: a block of keys has cells all over the grid."""
    announce("sparse_attention_backward scattered order", (w, d))
    case = (2, w, 1, d, 128, 0.4, "position", False)
    qkv, rel, _, out_rows, dout, rows = T.inputs(5, 2, w, 1, d, "position", False)
    sigma = torch.randperm(w * w, generator=T.gen(6), device=DEV).to(torch.int32)
    out = torch.zeros(rows, d, dtype=BF, device=DEV)
    B.ssam_sparse_attention(qkv, *rel, sigma, w, 128, 0.4, out=out)
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, 128, 0.4, out, dout)
    against_64_bits(case, (qkv, rel, sigma, None, dout, out), got)


@pytest.mark.parametrize("case", [(1, 14, 2, 64, 32, 0.5, "position", False), (1, 14, 2, 80, 32, 1.0, "content", False), (1, 32, 2, 64, 128, 0.6, "position", False),
                                  (1, 50, 1, 80, 128, 0.4, "content", False)])
def test_scores_that_grow(case):
    """Keys ten times as large at the end as at the start: the largest score of a query is found late, again and again, and few keys have all the weight.  Biases are
    small, so that their fp16 adds nothing to what the bounds hold."""
    announce("sparse_attention_backward growing scores", case)
    groups, w, h, d, tile, r, order, drop = case
    qkv, rel, sigma, out_rows, dout, rows = T.inputs(8, groups, w, h, d, order, drop, rel_std=0.01)
    qkv[:, :, 1] = (qkv[:, :, 1].float() * torch.linspace(0.5, 5.0, w * w, device=DEV)[None, :, None, None]).to(BF)
    out = torch.zeros(rows, h * d, dtype=BF, device=DEV)
    B.ssam_sparse_attention(qkv, *rel, sigma, w, tile, r, out=out)
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, dout)
    against_64_bits(case, (qkv, rel, sigma, None, dout, out), got)


@pytest.mark.parametrize("case", [(1, 4, 1, 16, 32, 1.0, "content", False), (1, 14, 1, 32, 32, 0.5, "position", False), (1, 17, 1, 64, 128, 0.4, "content", False)])
def test_against_differences(case):
    """Along directions, <gradient, direction> is the slope of sum(out * dout), out in 64 bits.  What it may be off by: the elements' bounds times the direction's
    elements, added up; the difference itself by 1e-5 of the sum of its products (a step of 1e-4 squared, times a third derivative below 1e3)."""
    announce("sparse_attention_backward differences", case)
    groups, w, h, d, tile, r, order, drop = case
    (qkv, rel, sigma, out_rows, dout, out), (dqkv, *drel) = T.run(case, seed=12)
    grads, size, dref, dsize = T.reference(qkv, *rel, sigma, w, tile, r, dout, None, d ** -0.5)
    seen, s = T.mask(w * w, tile, r), (sigma[0] if sigma.dim() == 2 else sigma).long()
    leaves = [qkv[0, :, i, 0].double() for i in range(3)] + [t.double() for t in rel]
    mine = [dqkv[0, :, i, 0].double() for i in range(3)] + [t.double() for t in drel]
    bounds = [2.0 ** -8 * a.abs() + 6 * 2.0 ** -9 * b for a, b in zip([grads[0, :, i, 0] for i in range(3)] + dref, [size[0, :, i, 0] for i in range(3)] + dsize)]

    def value(shift):
        moved = [a + b for a, b in zip(leaves, shift)]
        return (T.forward64(*moved, s, w, seen, d ** -0.5)[1] * dout.double().view(-1, d)).sum()

    g = T.gen(13)
    for leaf in range(5):
        for kind in range(2):
            u = [torch.zeros_like(t) for t in leaves]
            u[leaf] = torch.randn(leaves[leaf].shape, generator=g, device=DEV, dtype=torch.float64) if kind else mine[leaf] / mine[leaf].norm()
            step = 1e-4
            slope = (value([step * t for t in u]) - value([-step * t for t in u])) / (2 * step)
            got, off = (mine[leaf] * u[leaf]).sum(), (bounds[leaf] * u[leaf].abs()).sum() + 1e-5 * (mine[leaf] * u[leaf]).abs().sum()
            assert abs(got - slope) <= off, (leaf, kind, float(got), float(slope), float(off))


@pytest.mark.parametrize("case", [(3, 14, 2, 80, 32, 0.5, "content", True), (2, 17, 1, 64, 128, 0.4, "position", True), (1, 64, 1, 32, 128, 0.2, "position", True)])
def test_what_no_gradient_comes_from(case):
    """NaN in q and out of dropped queries, in rows of out and dout that no query has, and all over the workspace: nothing of it is seen."""
    announce("sparse_attention_backward NaN", case)
    groups, w, h, d, tile, r, order, drop = case
    (qkv, rel, sigma, out_rows, dout, out), want = T.run(case, seed=21)
    dropped = out_rows < 0
    assert dropped.any()
    bad = qkv.clone()
    bad[:, :, 0][dropped] = math.nan
    unused = torch.ones(out.shape[0], dtype=torch.bool, device=DEV)
    unused[out_rows[~dropped].long()] = False
    for t in (out, dout):
        t[unused] = math.nan
    n = B.ssam_sparse_attention_backward_workspace_bytes(groups, w * w, w, h, d)
    for fill in (0xff, 0x7c, 0x00):
        ws = torch.full((n,), fill, dtype=torch.uint8, device=DEV)
        got = B.ssam_sparse_attention_backward(bad, *rel, sigma, w, tile, r, out, dout, out_rows=out_rows, workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), hex(fill)
    assert (want[0][:, :, 0][dropped] == 0).all()


@pytest.mark.parametrize("w,tile,d", [(14, 32, 64), (14, 32, 80), (5, 128, 16), (28, 128, 64), (64, 128, 32)])
def test_rows_of_any_stride(w, tile, d):
    """q, k, v and their gradients in rows of their own strides, behind one another or apart: the same bits, and nothing between the rows is touched."""
    announce("sparse_attention_backward strides", (w, tile, d))
    groups, h, S = 2, 3, w * w
    case = (groups, w, h, d, tile, 0.5, "content", False)
    (qkv, rel, sigma, _, dout, out), (want, wh, ww) = T.run(case, seed=30)
    rs, gs, n = h * d + 24, h * d + 40, groups * S
    src = [torch.full((n, rs), math.nan, dtype=BF, device=DEV) for _ in range(3)]
    dst = [torch.full((n + 1, gs), 7.0, dtype=BF, device=DEV) for _ in range(3)]
    for i in range(3):
        src[i][:, :h * d] = qkv[:, :, i].reshape(n, h * d)
    dh, dw = torch.empty_like(rel[0]), torch.empty_like(rel[1])
    ws = torch.empty(B.ssam_sparse_attention_backward_workspace_bytes(groups, S, w, h, d), dtype=torch.uint8, device=DEV)
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    rc = B.lib().ssam_sparse_attention_backward(*map(p, src), C.c_long(rs), p(rel[0]), p(rel[1]), p(sigma), C.c_long(S), p(out), p(dout), None, *map(p, dst), C.c_long(gs), p(dh), p(dw),
                                                groups, S, w, h, d, tile, C.c_double(0.5), C.c_float(d ** -0.5), p(ws), C.c_size_t(ws.numel()),
                                                C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    torch.cuda.synchronize()
    for i in range(3):
        assert torch.equal(dst[i][:n, :h * d], want[:, :, i].reshape(n, h * d))
        assert (dst[i][:, h * d:] == 7).all() and (dst[i][n] == 7).all()
    assert torch.equal(dh, wh) and torch.equal(dw, ww)


def test_binding_refuses_shapes():
    (qkv, rel, sigma, _, dout, out), _ = T.run((2, 5, 2, 16, 32, 0.5, "content", False), seed=1)
    call = B.ssam_sparse_attention_backward
    for bad in (lambda: call(qkv, rel[0][:-1], rel[1], sigma, 5, 32, 0.5, out, dout), lambda: call(qkv, *rel, sigma[:, :-1].contiguous(), 5, 32, 0.5, out, dout),
                lambda: call(qkv, *rel, sigma, 5, 32, 0.5, out[:-1], dout[:-1]), lambda: call(qkv, *rel, sigma, 5, 32, 0.5, out, dout[:-1]),
                lambda: call(qkv, *rel, sigma, 5, 32, 0.5, out, dout, dqkv=torch.empty_like(qkv[:1])),
                lambda: call(qkv, *rel, sigma, 5, 32, 0.5, out, dout, out_rows=torch.zeros(3, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.SsamError):
        call(qkv, *rel, sigma, 5, 64, 0.5, out, dout)
    with pytest.raises(B.SsamError):
        call(qkv, *rel, sigma, 5, 32, 0.5, out, dout, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("case", [(3, 14, 2, 64, 32, 0.5, "content", True), (1, 28, 2, 64, 128, 0.4, "position", False), (1, 64, 2, 80, 128, 0.3, "position", False)])
def test_on_another_stream_and_in_a_graph(case):
    """Two calls at once on streams of their own, and captured, replayed three times with eager work between."""
    announce("sparse_attention_backward stream and graph", case)
    groups, w, h, d, tile, r, order, drop = case
    (qkv, rel, sigma, out_rows, dout, out), want = T.run(case, seed=40)
    dqkv = torch.empty_like(qkv)
    ws = torch.empty(B.ssam_sparse_attention_backward_workspace_bytes(groups, w * w, w, h, d), dtype=torch.uint8, device=DEV)

    def step(to=None, space=None):
        return B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, dout, out_rows=out_rows, dqkv=to, workspace=space)

    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for side in sides:
        with torch.cuda.stream(side):
            got.append(step())
    for side in sides:
        side.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
    with torch.cuda.stream(sides[0]):
        step(dqkv, ws)
    sides[0].synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(dqkv, ws)
    for turn in range(3):
        ws.fill_(255)
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
        assert all(torch.equal(a, b) for a, b in zip(step(), want)), turn
        torch.cuda.synchronize()


@pytest.mark.parametrize("w,tile,r,drop", [(7, 32, 0.5, True), (32, 128, 0.4, False)])
def test_a_block_both_ways(w, tile, r, drop):
    """The gradient calls as a training step takes them: LayerNorm of gathered rows, qkv, attention over groups, a contraction and GELU kept in 8 bits, and back to the stream's
    gradient and those of the LayerNorm's weights and both tables, against the same in 64 bits by automatic differentiation.  By norms: ten tensors on the way are
    rounded to bf16 (2^-9 each, of which no step makes more than twice as much), and 8 bits of 64 normal values (amax of 2.5, steps of 1/127 of it, off by 0.0057 at the root of the
    mean square) change GELU's slope by as much again: 20 * 2^-9 + 0.0114 is 0.05."""
    announce("gradients of a block", (w, tile, r, drop))
    g = T.gen(50)
    S, h, d, D, groups = w * w, 2, 64, 128, 3
    x = T.normal(g, groups, S, D, dtype=BF)
    order = torch.stack([torch.randperm(S, generator=g, device=DEV) for _ in range(groups)]).to(torch.int32)
    idx = order.clone()
    if drop:                                   # rows of padding: none of x's, and their queries' results are dropped
        idx[:, ::7] = -1
    out_rows = torch.where(idx >= 0, torch.arange(groups, device=DEV, dtype=torch.int32)[:, None] * S + idx, -1).to(torch.int32).contiguous()
    gamma, beta = T.normal(g, D, std=0.2) + 1, T.normal(g, D, std=0.2)
    Wq, W1 = T.normal(g, D, 3 * h * d, std=D ** -0.5, dtype=BF), T.normal(g, h * d, 192, std=2 * (h * d) ** -0.5, dtype=BF)
    rel = [T.normal(g, 2 * w - 1, d, std=0.1, dtype=BF) for _ in range(2)]
    da = T.normal(g, groups * S, 192, std=0.02, dtype=BF)
    mm = lambda a, b: (a.float() @ b.float()).to(BF)  # noqa: E731

    y = B.ssam_ln_gather(x, idx, S, gamma, beta, 1e-6, S)
    qkv = mm(y.view(-1, D), Wq).view(groups, S, 3, h, d)
    out = torch.zeros(groups * S, h * d, dtype=BF, device=DEV)
    B.ssam_sparse_attention(qkv, *rel, order, w, tile, r, out=out, out_rows=out_rows)
    a, codes, scales = B.ssam_gelu_checkpoint(mm(out, W1))

    dh, again = B.ssam_gelu_backward(codes, scales, da)
    dout = mm(dh, W1.T)
    dqkv, drh, drw = B.ssam_sparse_attention_backward(qkv, *rel, order, w, tile, r, out, dout, out_rows=out_rows)
    dy = mm(dqkv.view(-1, 3 * h * d), Wq.T).view(groups, S, D)
    dx, dgamma, dbeta = B.ssam_ln_gather_backward(x, idx, S, gamma, 1e-6, dy)

    leaf = [t.double().cpu().requires_grad_() for t in (x, gamma, beta, *rel)]
    seen, results = T.mask(S, tile, r).cpu(), []
    for i in range(groups):
        at = idx[i].long().cpu()
        rows = torch.nn.functional.layer_norm(leaf[0][i][at.clamp(min=0)], (D,), leaf[1], leaf[2], 1e-6) * (at >= 0)[:, None]
        f = (rows @ Wq.double().cpu()).view(S, 3, h, d)
        o = torch.cat([T.forward64(*(f[:, n, k] for n in range(3)), leaf[3], leaf[4], order[i].long().cpu(), w, seen, d ** -0.5)[1] for k in range(h)], 1)
        result = torch.zeros(S, h * d, dtype=torch.float64)
        keep = at >= 0
        results.append(result.index_copy(0, at[keep], o[keep]))
    u = torch.cat(results) @ W1.double().cpu()
    act = 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    (act * da.double().cpu()).sum().backward()
    for name, got, ref in (("gelu", a, act.detach()), ("gelu again", again, act.detach()), ("dx", dx, leaf[0].grad), ("dgamma", dgamma, leaf[1].grad), ("dbeta", dbeta, leaf[2].grad),
                           ("drel_h", drh, leaf[3].grad), ("drel_w", drw, leaf[4].grad)):
        got = got.double().cpu().view(ref.shape)
        off = float((got - ref).norm() / ref.norm())
        print(f"[parity] {name}: {off:.2e}", flush=True)
        assert torch.isfinite(got).all() and off <= 0.05, name
