"""Rows in 8 bits and their products through the C ABI, against whole-number arithmetic and 64 bits."""
import numpy as np
import pytest
import torch

import residual_reference as R
from helpers import announce
from paper_2605_17633_amd import binding as B
from test_linear_i8_forms import CASES, FORMS

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("rows,D", [(1, 16), (1, 1280), (3, 144), (65, 512), (7, 528), (33, 1024), (5, 1536), (9, 2048), (4, 2064), (13, 5120), (2, 5136), (3, 20000), (1, 131056), (4099, 64)])
def test_quantize(rows, D):
    announce("quantize_rows", rows, D)
    gen = torch.Generator().manual_seed(rows * 7 + D)
    x = (torch.randn(rows, D, generator=gen) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=gen).float())).to(BF)
    x[0, :3] = torch.tensor([127.0, 63.5, -64.5]) * float(x[0].abs().max().clamp(min=2.0 ** -20).log2().ceil().exp2())      # ties
    if rows > 2:
        x[1] = 0
        x[2] = x[2] * 2.0 ** -100 * 2.0 ** -20
    codes, scales = B.ssam_quantize_rows(x.to(DEV))
    want, want_scales = R.quantised(x.double().numpy())
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), want_scales)


def test_quantize_every_value_under_every_largest():
    """All bf16 magnitudes of 8 bits of mantissa under every largest mantissa: codes are the definition's."""
    tops = torch.arange(128, 256).float()
    x = torch.zeros(128, 528)
    x[:, 0] = tops
    for i, e in enumerate((1.0, 0.5, 0.25, 0.125)):
        x[:, 1 + 128 * i:1 + 128 * (i + 1)] = torch.minimum(torch.arange(128, 256).float() * e, tops[:, None]) * (1 - 2 * (torch.arange(128) % 2))
    codes, scales = B.ssam_quantize_rows(x.to(BF).to(DEV))
    want, want_scales = R.quantised(x.double().numpy())
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), want_scales)


def test_quantize_rows_that_are_not_finite():
    x = torch.randn(4, 2576, generator=torch.Generator().manual_seed(0)).to(BF)
    x[1, 2575], x[3, 0] = float("nan"), float("-inf")
    codes, scales = B.ssam_quantize_rows(x.to(DEV))
    assert torch.isnan(scales).tolist() == [False, True, False, True] and not codes[[1, 3]].any()
    want, want_scales = R.quantised(x[[0, 2]].double().numpy())
    assert np.array_equal(codes[[0, 2]].cpu().numpy(), want) and np.array_equal(scales[[0, 2]].cpu().numpy(), want_scales)


def _problem(M, N, K, seed, lo=-127):
    gen = torch.Generator().manual_seed(seed)
    codes = lambda *s: torch.randint(lo, 128, s, generator=gen).to(torch.int8)  # noqa: E731
    f = lambda n: torch.rand(n, generator=gen) * 0.02 + 0.001  # noqa: E731
    return codes(M, K), f(M), codes(N, K), f(N) / K ** 0.5, torch.randn(N, generator=gen)


def _reference(A, sa, W, sw, bias):
    """-> v in 64 bits, and what fp32 is off: the sum's rounding, two products' and the sum's with the bias"""
    acc = A.double() @ W.double().t()
    part = acc * sw.double() * sa.double()[:, None]
    v = part + bias.double()
    return v, R.U * (3 * part.abs() + v.abs()) * (1 + 4 * R.U)


def _gelu(v, err):
    """gelu_erf: its slope is 1.13 at most; erfc is off by 1.5e-7 and a dozen roundings, half of which t is multiplied by"""
    return torch.nn.functional.gelu(v), 1.13 * err + v.abs() * 0.5 * (1.5e-7 + 12 * R.U)


def _check(got, ref, err, what):
    got, allowed = got.double().cpu(), ref.abs() * R.BF + err * (1 + R.BF)
    off = (got - ref).abs()
    bad = off > allowed
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / (allowed + 1e-300)).max()):.2f} of what is allowed"


SIZES = [(1, 8, 16), (1, 1280, 1280), (2, 3840, 1280), (3, 576, 144), (5, 72, 48), (16, 264, 5120), (17, 1280, 640), (31, 120, 4096), (33, 2304, 768), (64, 64, 64), (65, 200, 272), (100, 1288, 1040),
         (127, 128, 128), (128, 384, 1152), (129, 136, 656), (200, 1280, 5120), (255, 520, 576), (257, 1152, 288), (313, 4096, 1024), (612, 576, 2304), (1000, 1000, 400), (1638, 1280, 2560),
         (2049, 264, 784), (4900, 576, 144), (5000, 8, 16), (7, 5120, 10240), (4096, 2304, 768), (3000, 3840, 1280)]


@pytest.mark.parametrize("M,N,K", SIZES, ids=str)
def test_linear(M, N, K):
    announce("linear_i8", M, N, K)
    A, sa, W, sw, bias = _problem(M, N, K, M + N + K)
    v, err = _reference(A, sa, W, sw, bias)
    d = [t.to(DEV) for t in (A, sa, W, sw, bias)]
    _check(B.ssam_linear_i8(*d), v, err, "bias")
    _check(B.ssam_linear_i8(*d, epilogue=B.EPI_BIAS_GELU), *_gelu(v, err), "gelu")
    # a map of images: slots without a token, entries past the last row, rows of C that nothing is written to
    gen = torch.Generator().manual_seed(M)
    per = max(1, -(-M // 3))
    tokens, batches = per + 3, -(-M // per)
    rows = torch.full((batches, per), -1, dtype=torch.int32)
    for b in range(batches):
        rows[b] = torch.randperm(tokens, generator=gen)[:per]
        if per > 2:
            rows[b, :2] = torch.tensor([-1, tokens])
    old = torch.randn(batches * tokens, N, generator=gen).to(BF)
    for epi in (B.EPI_BIAS_SCATTER, B.EPI_BIAS_SCATTER_ADD):
        ref, off, new = old.double(), torch.zeros(old.shape, dtype=torch.float64), torch.zeros(len(old), dtype=torch.bool)
        m = rows.view(-1)[:M].long()
        there = (m >= 0) & (m < tokens)
        to = (torch.arange(M) // per * tokens + m)[there]
        ref[to] = v[there] + (ref[to] if epi == B.EPI_BIAS_SCATTER_ADD else 0)
        off[to] = err[there] + R.U * ref[to].abs()
        new[to] = True
        got = B.ssam_linear_i8(*d, old.to(DEV), epilogue=epi, row_map=rows.to(DEV), rows_per_batch=per, map_batch_stride=per, dst_rows_per_batch=tokens)
        assert torch.equal(got.cpu()[~new], old[~new])
        _check(got.cpu()[new], ref[new], off[new], "mapped")


def _forced(form, epi, A, sa, W, sw, bias, C, rows):
    """A call with its form forced (None: its own), from tensors of the device; rows: the map of the epilogues that have one."""
    (M, K), N = A.shape, W.shape[0]
    args = (A.data_ptr(), K, sa.data_ptr(), W.data_ptr(), K, sw.data_ptr(), bias.data_ptr(), C.data_ptr(), N, M, N, K, epi, rows.data_ptr(), M, M, len(C))
    stream = torch.cuda.current_stream().cuda_stream
    rc = B.lib().ssam_linear_i8(*args, stream) if form is None else B.lib().ssam_linear_i8_as(*args, form, stream)
    assert rc == B.OK


def _forms_agree(M, N, K, epi, forms, against=32):
    gen = torch.Generator(device=DEV).manual_seed(M + N + K)
    codes = lambda *s: torch.randint(-128, 128, s, generator=gen, device=DEV, dtype=torch.int8)  # noqa: E731
    f = lambda n: torch.rand(n, generator=gen, device=DEV) * 0.02 + 0.001  # noqa: E731
    t = codes(M, K), f(M), codes(N, K), f(N) / K ** 0.5, torch.randn(N, generator=gen, device=DEV)
    mapped = epi in (B.EPI_BIAS_SCATTER, B.EPI_BIAS_SCATTER_ADD)
    rows = torch.randperm(M + 2, generator=gen, device=DEV)[:M].to(torch.int32)
    rows[torch.rand(M, generator=gen, device=DEV) < 0.1] = -1
    old = torch.randn(M + 2 if mapped else M, N, generator=gen, device=DEV).to(BF)
    want = old.clone()
    _forced(against, epi, *t, want, rows)
    for form in forms:
        got = old.clone()
        _forced(form, epi, *t, got, rows)
        assert torch.equal(got, want), (form, M, N, K, epi)
    return t, want


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forms_in_their_place(case):
    """The kernel that a call takes by itself: the bits of the one for few rows (sums are exact, and the rest is done alike)."""
    form, epi, M, N, K = case
    announce("linear_i8 form", *case)
    assert B.lib().ssam_linear_i8_form(M, N, K, epi) == form
    (A, sa, W, sw, bias), want = _forms_agree(M, N, K, epi, [None])
    if epi == B.EPI_BIAS:
        v = (A.double() @ W.double().t()) * sw.double() * sa.double()[:, None]
        err = R.U * (3 * v.abs() + (v + bias.double()).abs()) * (1 + 4 * R.U)
        _check(want, (v + bias.double()).cpu(), err.cpu(), "few rows")


@pytest.mark.parametrize("epi", range(4))
@pytest.mark.parametrize("M,N,K", [(1, 8, 16), (70, 72, 128), (257, 264, 144), (300, 520, 272), (513, 200, 400), (129, 776, 656), (390, 392, 784), (700, 1032, 1168), (1100, 1000, 48)])
def test_forms_outside_their_place(M, N, K, epi):
    """Every kernel on sizes that are no multiple of its tile, and on fewer slabs of K than its ring holds."""
    announce("linear_i8 forms", M, N, K, epi)
    _forms_agree(M, N, K, epi, [f for f in FORMS if f != 32])


def test_sums_are_exact():
    """The largest sums of 32 bits, and sums whose terms cancel to one: v is whole, so it comes out to half a step of bf16."""
    for K in (131056, 65536, 16):
        A = torch.full((3, K), -128, dtype=torch.int8)
        W = torch.full((16, K), -128, dtype=torch.int8)
        W[8:] = 127
        A[2, K // 2:], W[1, K // 2:] = 127, 127
        A[1, : K // 2] = 127
        W[3] = torch.where(torch.arange(K) % 2 == 0, 127, -127).to(torch.int8)
        W[3, 0] = 126
        one = lambda n: torch.ones(n, device=DEV)  # noqa: E731
        got = B.ssam_linear_i8(A.to(DEV), one(3), W.to(DEV), one(16), torch.zeros(16, device=DEV))
        _check(got, A.double() @ W.double().t(), (A.double() @ W.double().t()).abs() * 3 * R.U, f"K={K}")


def test_rows_do_not_depend_on_each_other():
    """A row alone, among few and among many: the same bits (sums are exact, and the rest is done alike)."""
    A, sa, W, sw, bias = (t.to(DEV) for t in _problem(3000, 1288, 656, 5))
    want = B.ssam_linear_i8(A, sa, W, sw, bias, epilogue=B.EPI_BIAS_GELU)
    for first, n in ((0, 1), (7, 3), (64, 17), (100, 150), (2000, 700)):
        got = B.ssam_linear_i8(A[first:first + n], sa[first:first + n].clone(), W, sw, bias, epilogue=B.EPI_BIAS_GELU)
        assert torch.equal(got, want[first:first + n]), (first, n)


@pytest.mark.parametrize("M,N,K", [(1, 72, 80), (20, 264, 208), (200, 520, 336), (700, 1288, 1040)])
def test_strides_and_what_lies_around(M, N, K):
    """Column slices of wider tensors: what lies beside an operand is not used, what lies beside C not written."""
    A, sa, W, sw, bias = _problem(M, N, K, 11)
    wide = lambda t, pad: torch.full((t.shape[0], t.shape[1] + pad), 77, dtype=t.dtype, device=DEV)  # noqa: E731
    WA, WW, WC = wide(A, 48), wide(W, 112), torch.full((M + 2, N + 24), 3.0, dtype=BF, device=DEV)
    WA[:, 16:16 + K], WW[:, 32:32 + K] = A.to(DEV), W.to(DEV)
    C = WC[1:M + 1, 8:8 + N]
    B.ssam_linear_i8(WA[:, 16:16 + K], sa.to(DEV), WW[:, 32:32 + K], sw.to(DEV), bias.to(DEV), C)
    _check(C, *_reference(A, sa, W, sw, bias), "strided")
    WC[1:M + 1, 8:8 + N] = 3.0
    assert bool((WC == 3.0).all())


def test_scales_that_are_not_finite_reach_their_rows():
    A, sa, W, sw, bias = (t.to(DEV) for t in _problem(70, 64, 96, 3))
    sa[5], sw[9] = float("nan"), float("nan")
    y = B.ssam_linear_i8(A, sa, W, sw, bias)
    bad = torch.isnan(y)
    assert bad[5].all() and bad[:, 9].all() and int(bad.sum()) == 64 + 70 - 1


def test_refused_epilogue_arguments_on_the_device():
    A, sa, W, sw, bias = (t.to(DEV) for t in _problem(8, 16, 32, 4))
    C, rows = torch.zeros(8, 16, dtype=BF, device=DEV), torch.arange(8, dtype=torch.int32, device=DEV)
    for k in (dict(rows_per_batch=4, map_batch_stride=4, dst_rows_per_batch=5), dict(rows_per_batch=4, map_batch_stride=8, dst_rows_per_batch=4)):
        with pytest.raises(ValueError):          # C has too few rows; the map too few entries
            B.ssam_linear_i8(A, sa, W, sw, bias, C, epilogue=B.EPI_BIAS_SCATTER, row_map=rows, **k)


def test_stream_and_graph():
    """Quantised and multiplied on a stream of its own and captured; replays with new inputs between eager calls."""
    gen = torch.Generator().manual_seed(0)
    xs = [torch.randn(500, 768, generator=gen).to(BF).to(DEV) for _ in range(2)]
    w, sw = B.ssam_quantize_rows((torch.randn(2304, 768, generator=gen) * 0.02).to(BF).to(DEV))
    bias = torch.randn(2304, generator=gen).to(DEV)
    run = lambda x: B.ssam_linear_i8(*B.ssam_quantize_rows(x), w, sw, bias)  # noqa: E731
    want = [run(x) for x in xs]
    live = xs[0].clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = run(live)
        stream.synchronize()
        assert torch.equal(got, want[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = run(live)
    for turn in range(4):
        live.copy_(xs[turn % 2])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want[turn % 2]) and torch.equal(run(xs[1 - turn % 2]), want[1 - turn % 2])


def test_a_block_in_8_bits():
    """A block's second half as it is used: the branch joins the stream, whose kept tokens go through fc1 and fc2 in 8 bits and back into it, and the next block's
    windows come out in 8 bits for qkv.  Against the same in 64 bits from every call's own inputs (each step's output is the next one's input), whole against whole too."""
    gen = torch.Generator().manual_seed(1)
    n = lambda *s, std=1.0: torch.randn(*s, generator=gen) * std  # noqa: E731
    Bn, g, D, Dm, K = 2, 20, 256, 1024, 160
    N = g * g
    table = torch.from_numpy(B.ssam_build_window_table(g, 14, 4)).to(DEV)
    slots = table.numel()
    keep = torch.stack([torch.randperm(N, generator=gen)[:K].sort()[0] for _ in range(Bn)]).to(torch.int32).to(DEV)
    windows, kept = B.ssam_invert_rows(table, N), B.ssam_invert_rows(keep, N)
    x, o = n(Bn, N, D).to(BF).to(DEV), n(Bn, slots, D).to(BF).to(DEV)
    norm = lambda: ((1 + n(D, std=0.1)).to(DEV), n(D, std=0.1).to(DEV))  # noqa: E731
    post, pre, post2, pre2, gates = norm(), norm(), norm(), norm(), [n(D, std=0.2).to(DEV), n(Bn, D, std=0.2).to(DEV)]
    weight = lambda rows, cols: (*B.ssam_quantize_rows(n(rows, cols, std=cols ** -0.5).to(BF).to(DEV)), n(rows, std=0.1).to(DEV))  # noqa: E731
    w1, w2, qkv = weight(Dm, D), weight(D, Dm), weight(3 * D, D)
    x1, c1, s1 = B.ssam_residual_norm_i8(x, o, windows, post, gates[0], 1.0, pre, kept, Ny=K)
    h = B.ssam_linear_i8(c1.view(-1, D), s1.view(-1), *w1, epilogue=B.EPI_BIAS_GELU)
    c2, s2 = B.ssam_quantize_rows(h)
    branch = B.ssam_linear_i8(c2, s2, *w2).view(Bn, K, D)
    x2, c3, s3 = B.ssam_residual_norm_i8(x1, branch, kept, post2, gates[1], 0.9375, pre2, windows, Ny=slots)
    y = B.ssam_linear_i8(c3.view(-1, D), s3.view(-1), *qkv).view(Bn, slots, 3 * D)

    f = lambda t: tuple(map(f, t)) if isinstance(t, tuple) else t.double().cpu()  # noqa: E731
    held = lambda w: f(w[0]) * f(w[1])[:, None]  # noqa: E731

    def eight(t):
        top = t.abs().amax(-1, keepdim=True)
        return torch.where(top > 0, torch.round(t * 127 / top) * top / 127, 0.0)

    k, win = keep.long().cpu(), table.long().cpu()
    r1 = R.step(f(x), f(o), windows.cpu(), f(post), f(gates[0]), 1.0, 1e-6)[0]
    u = (R.layer_norm(r1, 1e-6)[0] * f(pre[0]) + f(pre[1])).gather(1, k[..., None].expand(-1, -1, D))
    hidden = torch.nn.functional.gelu(eight(u) @ held(w1).t() + f(w1[2]))
    r2 = R.step(r1, eight(hidden) @ held(w2).t() + f(w2[2]), kept.cpu(), f(post2), f(gates[1]), 0.9375, 1e-6)[0]
    u = (R.layer_norm(r2, 1e-6)[0] * f(pre2[0]) + f(pre2[1]))[:, win.clamp(min=0)] * (win >= 0)[:, None]
    ref = eight(u) @ held(qkv).t() + f(qkv[2])
    # Rounded on its way: the stream twice, fc1's result and the branch (bf16: 2^-9.8 of a value's norm on average), and codes that fall to the other side of half a step where those
    # roundings move them (a step is top/127, near 3.5/127 of a deviation: moved by 2^-8 of a value, 1 in 10 by a whole step: 0.9 % of the norm), in three products.
    off = lambda got, want: float((f(got) - want).norm() / want.norm())  # noqa: E731
    announce("block in 8 bits", off(x2, r2), off(y, ref))
    assert off(x1, r1) <= R.BF and off(x2, r2) <= 1e-2 and off(y, ref) <= 2e-2
    pad = (win < 0)
    assert bool((y[:, pad] == qkv[2].to(BF)).all())


def test_tensors_past_32_bits():
    """Codes and results of more than 2^31 elements, and more rows than a launch takes: the last rows are what they are alone."""
    gen = torch.Generator(device=DEV).manual_seed(0)
    rows, D, tail = 1_100_000, 2048, 50
    x = torch.ones(rows, D, dtype=BF, device=DEV)
    x[-tail:] = torch.randn(tail, D, generator=gen, device=DEV).to(BF)
    codes, scales = B.ssam_quantize_rows(x)
    want, want_s = B.ssam_quantize_rows(x[-tail:].clone())
    assert torch.equal(codes[-tail:], want) and torch.equal(scales[-tail:], want_s) and bool((codes[:-tail:1000] == 127).all())
    del x
    w, sw = B.ssam_quantize_rows(torch.randn(2056, D, generator=gen, device=DEV).to(BF))
    bias = torch.randn(2056, generator=gen, device=DEV)
    y = B.ssam_linear_i8(codes, scales, w, sw, bias)
    assert y.numel() > 2 ** 31 and torch.equal(y[-tail:], B.ssam_linear_i8(want, want_s, w, sw, bias))
    del y, codes
    rows = (1 << 22) * 16 + 33
    x = torch.zeros(rows, 16, dtype=BF, device=DEV)
    x[-1] = torch.arange(16)
    codes, scales = B.ssam_quantize_rows(x)
    want = torch.from_numpy(R.quantised(np.arange(16.0)[None])[0][0]).to(DEV)
    assert torch.equal(codes[-1], want) and not codes[:-1].any() and bool((scales[:-1] == 2.0 ** -126).all())
    few = B.ssam_linear_i8(codes, scales, torch.ones(8, 16, dtype=torch.int8, device=DEV), torch.ones(8, device=DEV), torch.zeros(8, device=DEV))
    assert not few[:-1].any() and bool((few[-1] == few[-1, 0]).all()) and abs(float(few[-1, 0]) - float(want.int().sum()) * 15 / 127) <= 2.0 ** -8 * 120.5
