"""Gradients of Stripe-Sort attention against 64-bit arithmetic: every head size, windows and grids of one token and more, every order, dropped queries.

Tolerances.  Probabilities and their gradients dS are rounded to bf16 where they are multiplied (2^-9 of each at most; errors of the terms of a sum are
independent, so of a sum of n products that is 2^-9 of the root of the sum of their squares, and 6 times that is past what millions of them show), bias entries
to fp16 (2^-12 of a bias below 2; the tests' are), `out` to bf16 in delta, and the result to bf16: 2^-8 of the value."""
import math

import numpy as np
import pytest
import torch

from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def mask(S, tile, r):
    t = torch.arange(S, device=DEV) // tile
    ahead = min(-(-S // tile), int(math.floor(r * -(-S // tile) + 1e-6)))
    return (t[None, :] < ahead) | (t[None, :] == t[:, None])


def forward64(q, k, v, rel_h, rel_w, sigma, w, seen, scale):
    """[S, d] of one head in 64 bits -> the probabilities and the result"""
    row, col = sigma // w, sigma % w
    logits = q @ k.T * scale
    for rel, at in ((rel_h, row), (rel_w, col)):
        logits = logits + (q @ rel.T).gather(1, at[:, None] - at[None, :] + w - 1)
    p = torch.softmax(logits.masked_fill(~seen, -math.inf), 1)
    return p, p @ v


def reference(qkv, rel_h, rel_w, sigma, w, tile, r, dout, out_rows, scale):
    """-> gradients by the formulas in 64 bits, and for each the root of the sum of squares of the products that it is a sum of"""
    groups, S, _, h, d = qkv.shape
    seen = mask(S, tile, r)
    grads, size = torch.zeros(qkv.shape, dtype=torch.float64, device=DEV), torch.zeros(qkv.shape, dtype=torch.float64, device=DEV)
    rels = [rel_h.double(), rel_w.double()]
    drel, drel_size = [torch.zeros_like(t) for t in rels], [torch.zeros_like(t) for t in rels]
    for g in range(groups):
        s = (sigma[g] if sigma.dim() == 2 else sigma).long()
        for x in range(h):
            q, k, v = (qkv[g, :, i, x].double() for i in range(3))
            rows = torch.arange(g * S, g * S + S, device=DEV) if out_rows is None else out_rows.reshape(groups, S)[g].long()
            do = torch.where((rows >= 0)[:, None], dout.reshape(-1, h, d)[rows.clamp(min=0), x].double(), 0.0)
            p, o = forward64(q, k, v, *rels, s, w, seen, scale)
            dp = do @ v.T
            ds = p * (dp - (do * o).sum(1, keepdim=True))
            # delta is off by what the rounded result is: 2^-9 of the root of the sum of squares of dO * O
            near = (ds ** 2 + (p * (do ** 2 * o ** 2).sum(1, keepdim=True).sqrt()) ** 2).sqrt()
            dq, nq = ds @ k * scale, ((near ** 2) @ k ** 2) * scale ** 2
            for i, at in enumerate((s // w, s % w)):
                t = at[:, None] - at[None, :] + w - 1
                du, nu = (torch.zeros(S, 2 * w - 1, dtype=torch.float64, device=DEV).scatter_add_(1, t, m) for m in (ds, near ** 2))
                dq, nq = dq + du @ rels[i], nq + (nu + du ** 2) @ rels[i] ** 2            # G is rounded once more
                drel[i] += du.T @ q
                drel_size[i] += (nu + du ** 2).T @ q ** 2
            grads[g, :, 0, x], size[g, :, 0, x] = dq, nq.sqrt()
            grads[g, :, 1, x], size[g, :, 1, x] = ds.T @ q * scale, ((near ** 2).T @ q ** 2).sqrt() * scale
            grads[g, :, 2, x], size[g, :, 2, x] = p.T @ do, ((p ** 2).T @ do ** 2).sqrt()
    return grads, size, drel, [t.sqrt() for t in drel_size]


def check(got, ref, size, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    off = (got - ref).abs()
    bound = 2.0 ** -8 * ref.abs() + 6 * 2.0 ** -9 * size + 1e-30
    rel = float((got - ref).norm() / ref.norm().clamp(min=1e-300))
    print(f"[parity] {what}: off/bound {float((off / bound).max()):.3f}, norm {rel:.2e}", flush=True)
    assert (off <= bound).all(), f"{what}: {float((off / bound).max()):.3f} times the bound"


def inputs(seed, groups, w, h, d, order, drop, rel_std=0.1):
    g = gen(seed)
    S = w * w
    if order == "content":
        sigma = torch.stack([torch.randperm(S, generator=g, device=DEV) for _ in range(groups)]).to(torch.int32)
    else:
        sigma = torch.from_numpy(B.ssam_build_perm(w, w, 4 if S % 4 == 0 else 1)[0]).to(DEV)
    qkv = normal(g, groups, S, 3, h, d, std=0.7, dtype=BF)
    rel = [normal(g, 2 * w - 1, d, std=rel_std, dtype=BF) for _ in range(2)]
    out_rows = None
    rows = groups * S
    if drop:                              # some queries have no result, the others' lie anywhere in a larger tensor
        kept = torch.randperm(groups * S, generator=g, device=DEV)[:max(1, groups * S * 3 // 4)]
        rows = groups * S + 5
        out_rows = torch.full((groups * S,), -1, dtype=torch.int32, device=DEV)
        out_rows[kept] = torch.randperm(rows, generator=g, device=DEV)[:kept.numel()].to(torch.int32)
        out_rows = out_rows.view(groups, S)
    dout = normal(g, rows, h * d, std=0.02, dtype=BF)
    return qkv, rel, sigma, out_rows, dout, rows


def run(case, seed=0, **more):
    groups, w, h, d, tile, r, order, drop = case
    qkv, rel, sigma, out_rows, dout, rows = inputs(seed, groups, w, h, d, order, drop, **more)
    out = torch.zeros(rows, h * d, dtype=BF, device=DEV)
    B.ssam_sparse_attention(qkv, *rel, sigma, w, tile, r, out=out, out_rows=out_rows)
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, dout, out_rows=out_rows)
    return (qkv, rel, sigma, out_rows, dout, out), got


# (groups, side, heads, head size, mask tile, density, order, dropped queries)
CASES = [(1, 1, 1, 16, 32, 1.0, "position", False), (2, 1, 2, 64, 128, 0.5, "content", False), (3, 2, 1, 80, 32, 1.0, "position", True), (2, 5, 3, 32, 32, 0.4, "content", False),
         (4, 14, 2, 64, 32, 0.4, "position", False), (3, 14, 2, 80, 32, 0.5, "content", True), (2, 13, 1, 16, 32, 0.2, "content", True), (2, 12, 3, 32, 32, 1.0, "position", True),
         (1, 14, 4, 64, 32, 0.1, "content", False), (1, 11, 2, 80, 128, 0.5, "position", False), (2, 16, 2, 16, 128, 0.5, "position", False), (1, 17, 2, 64, 128, 0.4, "content", True),
         (1, 28, 2, 80, 128, 0.3, "position", False), (2, 28, 1, 64, 128, 1.0, "content", False), (1, 32, 2, 64, 128, 0.4, "position", True), (1, 33, 1, 32, 128, 0.6, "content", False),
         (1, 50, 1, 80, 128, 0.4, "content", False), (1, 64, 1, 64, 128, 0.4, "position", False), (1, 64, 1, 16, 128, 0.2, "content", True), (1, 65, 1, 64, 128, 0.2, "content", False),
         (1, 72, 1, 80, 128, 0.3, "position", False), (1, 66, 1, 32, 128, 0.5, "content", True)]


@pytest.mark.parametrize("case", CASES)
def test_gradients(case):
    announce("sparse_attention_backward", case)
    groups, w, h, d, tile, r, order, drop = case
    (qkv, rel, sigma, out_rows, dout, out), (dqkv, drel_h, drel_w) = run(case, seed=w)
    grads, size, drel, drel_size = reference(qkv, *rel, sigma, w, tile, r, dout, out_rows, d ** -0.5)
    for i, name in enumerate("qkv"):
        check(dqkv[:, :, i], grads[:, :, i], size[:, :, i], f"d{name} {case}")
    check(drel_h, drel[0], drel_size[0], "drel_h")
    check(drel_w, drel[1], drel_size[1], "drel_w")
    again = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, dout, out_rows=out_rows)
    assert all(torch.equal(a, b) for a, b in zip(again, (dqkv, drel_h, drel_w))), "another result for the same inputs"
    without, none, _ = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, dout, out_rows=out_rows, table_grads=False)
    assert torch.equal(without, dqkv) and none is None


def test_the_largest_grid():
    """128 x 128 tokens, one head: offsets, tables of 128 entries; the sums of the gradients along directions against 64 bits."""
    announce("sparse_attention_backward 128 x 128")
    case = (1, 128, 1, 64, 128, 0.1, "content", False)
    (qkv, rel, sigma, out_rows, dout, out), (dqkv, drel_h, drel_w) = run(case, seed=3)
    grads, size, drel, drel_size = reference(qkv, *rel, sigma, 128, 128, 0.1, dout, None, 0.125)
    for i, name in enumerate("qkv"):
        check(dqkv[:, :, i], grads[:, :, i], size[:, :, i], f"d{name}")
    check(drel_h, drel[0], drel_size[0], "drel_h")
    check(drel_w, drel[1], drel_size[1], "drel_w")
