"""Gradient calls at the edges of what they are documented to take: tables further apart than they are long, tensors past 2^31 elements, launches that are cut in pieces, and values
that are not finite, which reach what the formulas say and nothing else."""
import ctypes as C
import math

import pytest
import torch

import attention_gradient_reference as R
import test_gpu_attention_gradients as T
import test_gpu_gradients as G
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16


def raw(qkv, rel, sigma, stride, w, tile, r, out, dout):
    """The library's call with an order table of any stride, packed tensors."""
    groups, S, _, h, d = qkv.shape
    dqkv, drel = torch.empty_like(qkv), [torch.empty_like(t) for t in rel]
    ws = torch.empty(B.ssam_sparse_attention_backward_workspace_bytes(groups, S, w, h, d), dtype=torch.uint8, device=DEV)
    p = lambda t, i=0: C.c_void_p(t.data_ptr() + 2 * i * h * d)  # noqa: E731
    rc = B.lib().ssam_sparse_attention_backward(p(qkv), p(qkv, 1), p(qkv, 2), C.c_long(3 * h * d), p(rel[0]), p(rel[1]), p(sigma), C.c_long(stride), p(out), p(dout), None,
                                                p(dqkv), p(dqkv, 1), p(dqkv, 2), C.c_long(3 * h * d), p(drel[0]), p(drel[1]), groups, S, w, h, d, tile, C.c_double(r), C.c_float(d ** -0.5),
                                                p(ws), C.c_size_t(ws.numel()), C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    return dqkv, *drel


@pytest.mark.parametrize("w,tile", [(9, 32), (14, 128), (20, 128), (40, 128)])
def test_orders_further_apart(w, tile):
    announce("sparse_attention_backward orders further apart", w, tile)
    (qkv, rel, sigma, _, dout, out), want = T.run((3, w, 2, 32, tile, 0.5, "content", False), seed=60)
    apart = torch.full((3, w * w + 37), -5, dtype=torch.int32, device=DEV)
    apart[:, :w * w] = sigma
    assert all(torch.equal(a, b) for a, b in zip(raw(qkv, rel, apart, w * w + 37, w, tile, 0.5, out, dout), want))


@pytest.mark.parametrize("case", [(2, 14, 3, 64, 32, 0.4, "content", False), (2, 14, 1, 80, 128, 0.5, "position", False), (1, 28, 2, 64, 128, 0.4, "position", False), (1, 64, 2, 80, 128, 0.4, "position", False),
                                  (2, 33, 1, 32, 128, 0.3, "content", False), (1, 32, 9, 64, 128, 0.5, "position", False)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_gradient_that_is_not_finite(case, value):
    """In dout of one query of the last group and head, behind the prefix: its dQ, dK and dV of the keys that it sees and the tables' gradients, no other bit."""
    announce("sparse_attention_backward not finite", case, value)
    groups, w, h, d, tile, r = case[:6]
    S = w * w
    (qkv, rel, sigma, _, dout, out), want = T.run(case, seed=61)
    i = S - 2
    bad = dout.clone()
    bad[(groups - 1) * S + i, (h - 1) * d + 3] = value
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, out, bad)
    t = torch.arange(S, device=DEV) // tile
    seen = (t < R.prefix(S, tile, r)) | (t == t[i])
    touched = torch.zeros(groups, S, 3, h, dtype=torch.bool, device=DEV)
    touched[-1, i, 0, -1] = True
    touched[-1, :, 1:, -1] = seen[:, None]
    assert torch.equal(got[0][~touched], want[0][~touched])
    assert not bool(torch.isfinite(got[0][-1, i, 0, -1]).any())
    assert not bool(torch.isfinite(got[0][-1, seen, 1, -1]).any())                       # dS of the query is not finite for any key, in dV one feature
    assert not bool(torch.isfinite(got[0][-1, seen, 2, -1, 3]).any())
    order = (sigma[-1] if sigma.dim() == 2 else sigma).long()
    for a, b, cell in zip(got[1:], want[1:], (order // w, order % w)):
        t = torch.arange(2 * w - 1, device=DEV)
        reached = torch.zeros(2 * w - 1, dtype=torch.bool, device=DEV)
        reached[(cell[i] - cell[seen] + w - 1)] = True
        assert not bool(torch.isfinite(a[reached]).any())
        beside = (t < cell[i]) | (t > cell[i] + w - 1)                                    # no key is there for it
        assert torch.equal(a[beside], b[beside])


@pytest.mark.parametrize("case", [(2, 14, 2, 80, 32, 0.4, "content", False), (1, 32, 2, 64, 128, 0.4, "position", False), (1, 50, 1, 80, 128, 0.3, "content", False)])
def test_a_result_or_a_key_that_is_not_finite(case):
    """NaN in out of one query: its delta, so all of its dS; dV, in which out is not, keeps its bits.  NaN in a key behind the prefix: P of the queries of its tile, and so their dQ, and dK and dV
    of the keys that they see; no other query's dQ."""
    announce("sparse_attention_backward result or key not finite", case)
    groups, w, h, d, tile, r = case[:6]
    S = w * w
    (qkv, rel, sigma, _, dout, out), want = T.run(case, seed=66)
    i = S - 2
    t = torch.arange(S, device=DEV) // tile
    seen = (t < R.prefix(S, tile, r)) | (t == t[i])
    bad = out.clone()
    bad[(groups - 1) * S + i, (h - 1) * d] = math.nan
    got = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, tile, r, bad, dout)[0]
    assert torch.equal(got[:, :, 2], want[0][:, :, 2])
    assert bool(got[-1, i, 0, -1].isnan().all()) and bool(got[-1, seen, 1, -1].isnan().all())
    assert int(got[:, :, :2].isnan().sum()) == d * (1 + int(seen.sum()))
    keys = qkv.clone()
    keys[-1, i, 1, -1, 1] = math.nan
    got = B.ssam_sparse_attention_backward(keys, *rel, sigma, w, tile, r, out, dout)[0]
    same = t == t[i]
    assert bool(got[-1, same, 0, -1].isnan().all()) and int(got[:, :, 0].isnan().sum()) == d * int(same.sum())
    assert bool(got[-1, seen, 1:, -1].isnan().all()) and int(got[:, :, 1:].isnan().sum()) == 2 * d * int(seen.sum())


def test_a_batch_past_32_bits():
    """200 images of 64 x 64, 16 heads of 80: 3.1e9 elements of q, k and v.  The first and the last image by themselves: dQ has the same bits, dK and dV (whose sums are cut elsewhere) the
    same to a rounding: 1.5 steps of bf16."""
    announce("sparse_attention_backward past 32 bits")
    groups, w, h, d = 200, 64, 16, 80
    S = w * w
    g = T.gen(62)
    qkv = torch.empty(groups, S, 3, h, d, dtype=BF, device=DEV)
    out, dout = (torch.empty(groups * S, h * d, dtype=BF, device=DEV) for _ in range(2))
    for i in range(0, groups, 8):
        qkv[i:i + 8] = T.normal(g, 8, S, 3, h, d, std=0.7, dtype=BF)
        dout[i * S:(i + 8) * S] = T.normal(g, 8 * S, h * d, std=0.02, dtype=BF)
    rel = [T.normal(g, 2 * w - 1, d, std=0.1, dtype=BF) for _ in range(2)]
    sigma = torch.from_numpy(B.ssam_build_perm(w, w, 4)[0]).to(DEV)
    B.ssam_sparse_attention(qkv, *rel, sigma, w, 128, 0.4, out=out)
    dqkv, drel_h, drel_w = B.ssam_sparse_attention_backward(qkv, *rel, sigma, w, 128, 0.4, out, dout)
    for i in (0, groups // 2 + 3, groups - 1):
        one, _, _ = B.ssam_sparse_attention_backward(qkv[i:i + 1], *rel, sigma, w, 128, 0.4, out[i * S:(i + 1) * S], dout[i * S:(i + 1) * S])
        assert torch.equal(one[0, :, 0], dqkv[i, :, 0])
        a, b = one[0, :, 1:].float(), dqkv[i, :, 1:].float()
        assert bool(((a - b).abs() <= 1.5 * 2.0 ** -7 * b.abs() + 1e-7).all())
    assert bool(torch.isfinite(drel_h).all()) and bool(torch.isfinite(drel_w).all())


@pytest.mark.parametrize("accumulate", [True, False])
def test_layernorm_tables_further_apart(accumulate):
    announce("ln_gather_backward tables further apart", accumulate)
    x, idx, gamma, dy, dx0 = G.ln_inputs(3, 50, 44, 200, True, 63)
    apart = torch.full((3, 61), 7, dtype=torch.int32, device=DEV)
    apart[:, :44] = idx
    want = B.ssam_ln_gather_backward(x, idx, 44, gamma, G.EPS, dy, dx=dx0.clone(), accumulate=accumulate)
    got = B.ssam_ln_gather_backward(x, apart, 61, gamma, G.EPS, dy, dx=dx0.clone(), accumulate=accumulate)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_layernorm_past_32_bits():
    """300 million rows of 8: 2.4e9 elements; rows at both ends and in the middle by themselves give the same bits."""
    announce("ln_gather_backward past 32 bits")
    n, D = 300 * 1000 * 1000, 8
    g = T.gen(64)
    x, dy = (torch.empty(1, n, D, dtype=BF, device=DEV) for _ in range(2))
    some = 10 * 1000 * 1000
    for i in range(0, n, some):
        x[0, i:i + some] = T.normal(g, some, D, dtype=BF)
        dy[0, i:i + some] = T.normal(g, some, D, std=0.02, dtype=BF)
    idx = torch.arange(n - 1, -1, -1, dtype=torch.int32, device=DEV)
    gamma = 1 + T.normal(g, D, std=0.2)
    dx, dgamma, dbeta = B.ssam_ln_gather_backward(x, idx, 0, gamma, G.EPS, dy)
    for i in (0, n // 2 - 500, n - 1000):
        at = torch.arange(999, -1, -1, dtype=torch.int32, device=DEV)
        one, _, _ = B.ssam_ln_gather_backward(x[:, i:i + 1000], at, 0, gamma, G.EPS, dy[:, n - i - 1000:n - i].contiguous())
        assert torch.equal(one[0], dx[0, i:i + 1000])
    # 146485 rows of a wave one after the other and 2048 waves: each sum is off by 2^-24 of the partial sums (random walks, a thousandth of the sum of magnitudes) a step
    total, size = dy[0].sum(0, dtype=torch.float64), dy[0].abs().sum(0, dtype=torch.float64)
    assert bool(((dbeta.double() - total).abs() <= 2.0 ** -24 * 146485 * 1e-3 * size).all()) and bool(torch.isfinite(dgamma).all())


@pytest.mark.parametrize("rows,D", [((1 << 27) + 3, 8), (3, 1 << 24), (1500, 1 << 20)])
def test_8_bits_in_pieces(rows, D):
    """More than 2^30 places of eight values: several launches.  (The last: 1.6e9 elements in rows of 2^20.)"""
    announce("checkpoint in pieces", rows, D)
    g = T.gen(65)
    x = torch.empty(rows, D, dtype=BF, device=DEV)
    flat = x.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device=DEV))
    a, codes, scales = B.ssam_gelu_checkpoint(x)
    back = B.ssam_checkpoint_restore(codes, scales)
    dh, again = B.ssam_gelu_backward(codes, scales, x)
    cut = (1 << 30) // (8 * -(-D // 64))                       # rows of a launch
    for r in {0, rows - min(rows, 3), *(i for i in range(cut - 2, rows, cut))}:
        at = slice(r, min(r + 4, rows))
        wa, wc, wsc = B.ssam_gelu_checkpoint(x[at].contiguous())
        wd, wag = B.ssam_gelu_backward(wc, wsc, x[at].contiguous())
        for got, want in ((a, wa), (codes, wc), (scales, wsc), (back, B.ssam_checkpoint_restore(wc, wsc)), (dh, wd), (again, wag)):
            assert torch.equal(got[at], want), r
