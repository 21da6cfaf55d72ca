"""The step between two halves of a block and its gradients through the C ABI, against formulas in 64 bits."""
import numpy as np
import pytest
import torch

import residual_reference as R
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, EPS = "cuda", 1e-6

# B, N, No, Ny, D, post, gate, pre, alpha, maps: every width's number of chunks a lane, every combination of norms and gates, maps of all images and of each,
# tokens without a branch, without a row of the result, and with neither
CASES = [
    (1, 1, 1, 1, 8, True, "features", True, 1.0, "own"),
    (2, 3, 3, 3, 16, True, "images", True, 0.5, "own"),
    (3, 37, 20, 11, 144, True, "features", True, 0.9375, "each"),
    (2, 64, 70, 80, 512, False, "images", True, 1.25, "shared"),
    (2, 50, 30, 50, 520, True, "none", True, -0.75, "each"),
    (1, 33, 40, 9, 768, False, "none", True, 1.0, "shared"),
    (4, 19, 19, 7, 1024, True, "images", False, 0.9375, "each"),
    (2, 25, 16, 30, 1280, True, "features", True, 0.9375, "each"),
    (2, 21, 30, 12, 1536, False, "features", False, 0.0, "shared"),
    (2, 17, 9, 17, 1544, True, "images", True, 0.9375, "each"),
    (1, 30, 15, 31, 2048, True, "features", True, 0.9375, "each"),
    (3, 12, 0, 9, 1280, False, "none", True, 1.0, "each"),               # no branch: a LayerNorm alone
    (2, 12, 6, 5, 256, True, "features", True, 0.9375, "empty"),          # maps that name nothing
    (300, 1, 1, 1, 64, True, "images", True, 0.9375, "own"),              # one token an image
]


def _map(gen, kind, B_, N, rows):
    """[N] or [B,N]: rows dealt to tokens, none twice; entries that name no row are -1 or past the last one."""
    if kind == "own":
        return None
    if kind == "empty":
        return torch.full((N,), -1, dtype=torch.int32)
    out = []
    for _ in range(B_ if kind == "each" else 1):
        m = torch.full((N,), -1)
        k = min(N, rows)
        k = max(1, k - k // 4)
        m[torch.randperm(N, generator=gen)[:k]] = torch.randperm(rows, generator=gen)[:k]
        m[(m < 0) & (torch.rand(N, generator=gen) < 0.3)] = rows
        out.append(m)
    return torch.stack(out).squeeze(0).to(torch.int32) if kind == "shared" or B_ == 1 else torch.stack(out).to(torch.int32)


def _inputs(case, seed):
    Bn, N, No, Ny, D, post, gate, pre, alpha, maps = case
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: torch.randn(*s, generator=gen) * std  # noqa: E731
    bf = lambda t: t.to(torch.bfloat16)  # noqa: E731
    s = {"x": bf(n(Bn, N, D) + n(D, std=0.5) + 0.5), "o": bf(n(Bn, No, D, std=0.7)) if No else None, "src": _map(gen, maps, Bn, N, No) if No else None,
         "post": (1 + n(D, std=0.2), n(D, std=0.2)) if post else None, "gate": None if gate == "none" else 0.5 + n(*((Bn, D) if gate == "images" else (D,)), std=0.3),
         "alpha": alpha, "pre": (1 + n(D, std=0.2), n(D, std=0.2)) if pre else None, "dst": _map(gen, maps, Bn, N, Ny) if pre else None,
         "dx_out": bf(n(Bn, N, D, std=0.1)), "dy": bf(n(Bn, Ny, D, std=0.1)) if pre else None}
    return s


def _dev(s):
    put = lambda v: v.to(DEV) if isinstance(v, torch.Tensor) else tuple(put(t) for t in v) if isinstance(v, tuple) else v  # noqa: E731
    return {k: put(v) for k, v in s.items()}


def _double(s):
    put = lambda v: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else tuple(put(t) for t in v) if isinstance(v, tuple) else v  # noqa: E731
    return {k: put(v) for k, v in s.items()}


def _within(got, ref, err, what, step=R.BF):
    """|got - ref| <= half a step of what is stored and what fp32 may be off (which the rounding may carry on by that much more)"""
    got, allowed = got.double().cpu(), (ref.abs() * step + err * (1 + step))
    off = (got - ref).abs()
    bad = off > allowed
    assert torch.isfinite(got).all() and not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / (allowed + 1e-300)).max()):.2f} of what is allowed"


STEP = ("o", "src", "post", "gate", "alpha", "pre", "dst")


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case):
    announce("residual_norm", case)
    s, Ny = _inputs(case, 1), case[3]
    d, r = _dev(s), _double(s)
    before = d["x"].clone()
    y0 = torch.full((case[0], Ny, case[4]), 3.0, dtype=torch.bfloat16, device=DEV) if s["pre"] else None
    x_out, y = B.ssam_residual_norm(d["x"], **{k: d[k] for k in STEP}, eps=EPS, y=y0)
    assert torch.equal(d["x"], before)
    ref, err = R.step(r["x"], r["o"], r["src"], r["post"], r["gate"], r["alpha"], EPS)
    _within(x_out, ref, err, "x_out")
    has = torch.zeros(case[:2], dtype=torch.bool) if s["o"] is None else R.rows_of(R.own_order(*case[:2]) if s["src"] is None else s["src"], r["o"], case[0])[1][..., 0]
    assert torch.equal(x_out.cpu()[~has], s["x"][~has])                       # bit for bit
    # in place: the same, and so is the second LayerNorm in 8 bits from it
    again, y2 = B.ssam_residual_norm(d["x"], **{k: d[k] for k in STEP}, eps=EPS, Ny=Ny, x_out=d["x"])
    assert again is d["x"] and torch.equal(again, x_out)
    if not s["pre"]:
        assert y is None and y2 is None
        return
    stored = x_out.cpu().double()
    want = R.layer_norm(stored, EPS)[0] * r["pre"][0] + r["pre"][1]
    off = R.layer_norm_error(stored, EPS) * r["pre"][0].abs() + 2 * R.U * (want.abs() + r["pre"][1].abs())
    m = (R.own_order(*case[:2]) if s["dst"] is None else s["dst"]).expand(case[0], -1).long()
    b, t = torch.nonzero((m >= 0) & (m < Ny), as_tuple=True)
    named = torch.zeros(case[0], Ny, dtype=torch.bool)
    named[b, m[b, t]] = True
    assert bool((y.cpu()[~named] == 3.0).all()) and bool((y2.cpu()[~named] == 0).all()) and torch.equal(y.cpu()[named], y2.cpu()[named])
    _within(y.cpu()[b, m[b, t]], want[b, t], off[b, t], "y")
    if case[4] % 16:
        return
    x8, codes, scales = B.ssam_residual_norm_i8(before, **{k: d[k] for k in STEP}, eps=EPS, Ny=Ny)
    assert torch.equal(x8, x_out)
    codes, scales = codes.cpu(), scales.cpu().double()
    assert not codes[~named].any() and not scales[~named].any()
    if not named.any():
        return
    assert bool((codes[named].int().abs().amax(1) == 127).all())
    want, off = want[b, t], off[b, t]
    held = codes[b, m[b, t]].double() * scales[b, m[b, t]][:, None]
    top = want.abs().amax(1, keepdim=True)
    # half a step of the scale; the scale's own error moves a code's value by up to all of the value's: the largest's error and four roundings
    allowed = top / 254 + off + (off.amax(1, keepdim=True) / top + 4 * R.U) * want.abs() * (1 + 1 / 127)
    assert bool(((held - want).abs() <= allowed * (1 + 1e-6)).all())


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradients(case):
    announce("residual_norm_backward", case)
    s = _inputs(case, 2)
    d, r = _dev(s), _double(s)
    do0 = torch.full_like(d["o"], 5.0) if s["o"] is not None else None
    args = {k: d[k] for k in (*STEP, "dy", "dx_out")}
    dx, do, dgate, dpost, dpre = B.ssam_residual_norm_backward(d["x"], **args, eps=EPS, do=do0)
    form = (r["x"], r["o"], r["src"], r["post"], r["gate"], r["alpha"], r["pre"], r["dst"], EPS, r["dy"], r["dx_out"])
    want, err = R.step_gradients(*form), R.step_gradient_errors(*form)
    _within(dx, want["dx"], err["dx"], "dx")
    if s["o"] is not None:
        m = (R.own_order(*case[:2]) if s["src"] is None else s["src"]).expand(case[0], -1).long()
        b, t = torch.nonzero((m >= 0) & (m < case[2]), as_tuple=True)
        named = torch.zeros(do.shape[:2], dtype=torch.bool)
        named[b, m[b, t]] = True
        assert bool((do.cpu()[~named] == 5.0).all())
        _within(do.cpu()[named], want["do"][named], err["do"][named], "do")
    for name, t in (("dgate", dgate), *((("dpost_g", dpost[0]), ("dpost_b", dpost[1])) if dpost else ()), *((("dpre_g", dpre[0]), ("dpre_b", dpre[1])) if dpre else ())):
        assert (t is None) == (name not in want)
        if t is not None:
            _within(t, want[name], err[name], name, step=R.U)
    # without the weights' gradients, and over dx_out
    dx2, do2, *none = B.ssam_residual_norm_backward(d["x"], **args, eps=EPS, dx=d["dx_out"], do=None if do0 is None else do0.clone(), weight_grads=False)
    assert none == [None, None, None] and torch.equal(dx2, dx) and (do is None or torch.equal(do2, do))


def test_gradients_without_what_comes_from_behind():
    case = CASES[7]
    s = _inputs(case, 3)
    d = _dev(s)
    args = {k: d[k] for k in (*STEP, "dy")}
    nothing = B.ssam_residual_norm_backward(d["x"], **args, eps=EPS)
    zeros = B.ssam_residual_norm_backward(d["x"], **args, eps=EPS, dx_out=torch.zeros_like(d["x"]))
    for a, b in zip((nothing[0], nothing[1], nothing[2], *nothing[3], *nothing[4]), (zeros[0], zeros[1], zeros[2], *zeros[3], *zeros[4])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("gate,N,D", [("features", 1500, 1280), ("images", 1500, 1280), ("features", 6000, 64), ("images", 6000, 144), ("features", 1400, 2048)])
def test_many_tokens_same_bits_and_workspace_bounds(gate, N, D):
    """More tokens than the waves of a launch; bytes around the workspace stay as they are; the same inputs give the same bits."""
    case = (3, N, 1000, 700, D, True, gate, True, 0.9375, "each")
    announce("residual_norm_backward", case)
    s = _inputs(case, 4)
    d, r = _dev(s), _double(s)
    need = B.ssam_residual_norm_backward_workspace_bytes(3, N, D, 3 if gate == "images" else 1)
    room = torch.full((need + 512,), 77, dtype=torch.uint8, device=DEV)
    args = {k: d[k] for k in (*STEP, "dy", "dx_out")}
    runs = [B.ssam_residual_norm_backward(d["x"], **args, eps=EPS, workspace=room[256:256 + need]) for _ in range(2)]
    assert bool((room[:256] == 77).all()) and bool((room[256 + need:] == 77).all())
    flat = lambda g: (g[0], g[1], g[2], *g[3], *g[4])  # noqa: E731
    assert all(torch.equal(a, b) for a, b in zip(*map(flat, runs)))
    form = (r["x"], r["o"], r["src"], r["post"], r["gate"], r["alpha"], r["pre"], r["dst"], EPS, r["dy"], r["dx_out"])
    want, err = R.step_gradients(*form), R.step_gradient_errors(*form)
    for name, t in zip(("dx", "do", "dgate", "dpost_g", "dpost_b", "dpre_g", "dpre_b"), flat(runs[0])):
        _within(t, want[name], err[name], name, step=R.BF if name in ("dx", "do") else R.U)


def test_rows_that_are_not_finite():
    """Infinity and NaN reach the rows that they are in, and no other; in 8 bits their scale is NaN."""
    case = (1, 6, 6, 6, 256, True, "features", True, 1.0, "own")
    d = _dev(_inputs(case, 5))
    d["x"][0, 1, 3], d["o"][0, 2, 200], d["o"][0, 4, 0] = float("inf"), float("nan"), float("-inf")
    x_out, y = B.ssam_residual_norm(d["x"], **{k: d[k] for k in STEP}, eps=EPS)
    _, codes, scales = B.ssam_residual_norm_i8(d["x"], **{k: d[k] for k in STEP}, eps=EPS)
    assert torch.isnan(y).all(2)[0].tolist() == [False, True, True, False, True, False]
    assert torch.isfinite(y).all(2)[0].tolist() == [True, False, False, True, False, True]
    assert torch.isnan(scales[0]).tolist() == [False, True, True, False, True, False] and not codes[0, [1, 2, 4]].any()
    assert torch.isinf(x_out[0, 1, 3]) and torch.isfinite(x_out[0, [0, 3, 5]]).all()


def test_constant_and_extreme_rows():
    """A row without deviation is its shift; rows of the largest numbers that squares hold, and of subnormal ones."""
    D = 768
    x = torch.zeros(1, 4, D, dtype=torch.bfloat16)
    x[0, 0] = 3.0
    x[0, 1] = torch.randn(D, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16) * 2.0 ** 55
    x[0, 2] = torch.randn(D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16) * 2.0 ** -126
    g, b = torch.ones(D), torch.linspace(-1, 1, D)
    _, y = B.ssam_residual_norm(x.to(DEV), pre=(g.to(DEV), b.to(DEV)), eps=EPS)
    v = x.double()
    want = R.layer_norm(v, EPS)[0] + b.double()
    _within(y, want, R.layer_norm_error(v, EPS) + 2 * R.U * (want.abs() + b.abs()), "y")


def test_invert_rows():
    table = torch.from_numpy(B.ssam_build_window_table(30, 14, 4)).to(DEV)
    inv = B.ssam_invert_rows(table, 900)
    assert torch.equal(table[inv.long()], torch.arange(900, dtype=torch.int32, device=DEV))
    keep = torch.stack([torch.randperm(901, generator=torch.Generator().manual_seed(i))[:300] for i in range(3)]).to(torch.int32)
    keep[0, 5], keep[1, 6] = -7, 1 << 30
    inv = B.ssam_invert_rows(keep.to(DEV), 900).cpu()
    want = np.full((3, 900), -1)
    for b in range(3):
        for p, t in enumerate(keep[b].tolist()):
            if 0 <= t < 900:
                want[b, t] = p
    assert np.array_equal(inv.numpy(), want)


def test_stream_and_graph():
    """On a stream of its own, and captured: replays with new inputs in place, between eager calls that use the same buffers' kin."""
    case = (2, 200, 150, 120, 1024, True, "images", True, 0.9375, "each")
    a, b = _dev(_inputs(case, 6)), _dev(_inputs(case, 7))
    b |= {"src": a["src"], "dst": a["dst"]}
    ws = torch.empty(B.ssam_residual_norm_backward_workspace_bytes(2, 200, 1024, 2), dtype=torch.uint8, device=DEV)

    def both(s, **k):
        x, y = B.ssam_residual_norm(s["x"], **{n: s[n] for n in STEP}, eps=EPS, Ny=120)
        g = B.ssam_residual_norm_backward(s["x"], **{n: s[n] for n in (*STEP, "dy", "dx_out")}, eps=EPS, **k)
        return x, y, g[0], g[1], g[2], *g[3], *g[4]

    want = [both(s) for s in (a, b)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    live = {k: v.clone() if isinstance(v, torch.Tensor) else tuple(t.clone() for t in v) if isinstance(v, tuple) else v for k, v in a.items()}
    with torch.cuda.stream(stream):
        got = both(live, workspace=ws)
        stream.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want[0]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = both(live, workspace=ws)
    for turn in range(4):
        s = (b, a)[turn % 2]
        for k, v in s.items():
            for to, t in zip(live[k] if isinstance(v, tuple) else [live[k]], v if isinstance(v, tuple) else [v]):
                if isinstance(t, torch.Tensor):
                    to.copy_(t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want[1 - turn % 2])), turn
        assert all(torch.equal(u, v) for u, v in zip(both(s), want[1 - turn % 2]))


def test_gradients_against_differences_of_the_call():
    """Differences of the forward call itself: y is rounded to bf16 (half a step of each value, either side), the rest is smaller by far."""
    case = (2, 16, 12, 14, 128, True, "images", True, 0.9375, "each")
    s = _inputs(case, 8)
    d = _dev(s)
    gen = torch.Generator().manual_seed(9)
    x_out, y = B.ssam_residual_norm(d["x"], **{k: d[k] for k in STEP}, eps=EPS, Ny=14)
    wy = torch.randn(y.shape, generator=gen).to(torch.bfloat16).to(DEV)
    grads = B.ssam_residual_norm_backward(x_out, **{k: d[k] for k in STEP}, eps=EPS, dy=wy)
    for name, got in (("gate", grads[2]), ("post", grads[3][0]), ("pre", grads[4][0])):
        t = d[name][0] if isinstance(d[name], tuple) else d[name]
        by = torch.randn(t.shape, generator=gen).to(DEV)
        h, sides = 0.25, []
        for sign in (1, -1):
            moved = t + sign * h * by
            k = {n: d[n] for n in STEP} | {name: (moved, d[name][1]) if isinstance(d[name], tuple) else moved}
            # the stream in front of the second LayerNorm is rounded to bf16 too: one more half step of each of its values, through 1 / deviation
            sides.append(B.ssam_residual_norm(d["x"], **k, eps=EPS, Ny=14)[1].double())
        diff = float((wy.double() * (sides[0] - sides[1])).sum()) / (2 * h)
        # roundings are independent: five deviations of the sum of both sides' (y, and the stream behind it), and h^2 of the third derivative
        noise = float((wy.double() ** 2 * (sides[0] ** 2 + sides[1] ** 2 + 2 * 3.0 ** 2)).sum()) ** 0.5 * R.BF / (2 * h)
        ref = float((got.double() * by.double()).sum())
        curve = 0.0 if name == "pre" else h * h * float((wy.double().abs().sum()))
        announce("differences", name, ref, diff, noise, curve)
        assert abs(ref - diff) <= 5 * noise + curve, name


def test_scales_are_of_the_row_alone():
    """A shift of the last features that is larger than every value of the row: lanes past the row have no say in its scale."""
    D = 1040
    x = torch.randn(1, 3, D, generator=torch.Generator().manual_seed(0)) * 0.1
    x[:, :, -8:] = -5.0
    g, b = torch.ones(D), torch.zeros(D)
    v = x.to(torch.bfloat16).double()
    b[-8:] = -R.layer_norm(v, EPS)[0][0, 0, -8:].float()               # those features come out near 0, far below the others
    _, codes, scales = B.ssam_residual_norm_i8(x.to(torch.bfloat16).to(DEV), pre=(g.to(DEV), b.to(DEV)), eps=EPS)
    want = R.layer_norm(v, EPS)[0] + b.double()
    top = want.abs().amax(2)
    assert float(b.abs().max()) > 2 * float(top.max())
    off = (R.layer_norm_error(v, EPS) + 2 * R.U * (want.abs() + b.double().abs())).amax(2) / 127 + 4 * R.U * top / 127
    assert bool(((scales.cpu().double() - top / 127).abs() <= off).all()) and bool((codes.int().abs().amax(2) == 127).all())


def test_tensors_past_32_bits():
    """More than 2^31 elements: the last tokens are what the same tokens are alone."""
    N, D, tail = 1_050_000, 2048, 40
    x, o = (torch.empty(1, N, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    gen = torch.Generator(device=DEV).manual_seed(0)
    for t in (x, o):
        t[:, :-tail] = 1.0
        t[:, -tail:] = torch.randn(1, tail, D, generator=gen, device=DEV).to(torch.bfloat16)
    norm = lambda: (1 + torch.randn(D, generator=gen, device=DEV) * 0.1, torch.randn(D, generator=gen, device=DEV) * 0.1)  # noqa: E731
    post, pre, gate = norm(), norm(), torch.rand(D, generator=gen, device=DEV)
    back = torch.arange(N - 1, -1, -1, dtype=torch.int32, device=DEV)                     # y in the other order: its first rows are the last tokens
    x_out, y = B.ssam_residual_norm(x, o, None, post, gate, 0.9375, pre, back)
    few = lambda t: t[:, -tail:].contiguous()  # noqa: E731
    want_x, want_y = B.ssam_residual_norm(few(x), few(o), None, post, gate, 0.9375, pre)
    assert torch.equal(few(x_out), want_x) and torch.equal(y[:, :tail].flip(1), want_y)
    _, codes, scales = B.ssam_residual_norm_i8(x, o, None, post, gate, 0.9375, pre, x_out=x_out)
    _, want_c, want_s = B.ssam_residual_norm_i8(few(x), few(o), None, post, gate, 0.9375, pre)
    assert torch.equal(few(codes), want_c) and torch.equal(scales[:, -tail:], want_s)
    del codes
    dx, do, *_ = B.ssam_residual_norm_backward(x_out, o, None, post, gate, 0.9375, pre, None, dy=x, dx_out=o, do=y)
    want = B.ssam_residual_norm_backward(few(x_out), few(o), None, post, gate, 0.9375, pre, None, dy=few(x), dx_out=few(o))
    assert torch.equal(few(dx), want[0]) and torch.equal(few(do), want[1])


def test_more_tokens_than_a_launch_takes():
    N = (1 << 26) + (1 << 22) * 16 + 21
    x = torch.ones(1, N, 8, dtype=torch.bfloat16, device=DEV)
    x[0, -1] = torch.arange(8)
    x[0, (1 << 22) * 16] = torch.arange(8)
    _, y = B.ssam_residual_norm(x, pre=(torch.ones(8, device=DEV), torch.zeros(8, device=DEV)))
    want = torch.nn.functional.layer_norm(torch.arange(8.0), (8,), eps=EPS).to(torch.bfloat16).to(DEV)
    named = torch.tensor([N - 1, (1 << 22) * 16], device=DEV)
    # (a step of bf16 is 2^-7 of the value; the row of ones has no deviation)
    assert torch.allclose(y[0, named].float(), want.float().expand(2, -1), rtol=2 ** -7, atol=0)
    assert int((y[0] != 0).any(1).sum()) == 2


def test_rows_that_no_token_names_are_not_read():
    """NaN in rows of the branch and of the gradient of y that no map names reaches nothing; outputs there stay as they were."""
    case = (2, 40, 60, 50, 264, True, "images", True, 0.9375, "each")
    d = _dev(_inputs(case, 10))
    args = {k: d[k] for k in (*STEP, "dy", "dx_out")}
    step = {k: d[k] for k in STEP}
    want = (*B.ssam_residual_norm(d["x"], **step, eps=EPS, Ny=50), *B.ssam_residual_norm_backward(d["x"], **args, eps=EPS))
    for name, which, rows in (("o", "src", 60), ("dy", "dst", 50)):
        named = torch.zeros(2, rows + 1, dtype=torch.bool, device=DEV)
        m = d[which].long()
        named.scatter_(1, torch.where((m >= 0) & (m < rows), m, rows), True)
        for t in (step, args):
            if name in t:
                t[name] = torch.where(named[:, :rows, None], t[name], float("nan"))
    got = (*B.ssam_residual_norm(d["x"], **step, eps=EPS, Ny=50), *B.ssam_residual_norm_backward(d["x"], **args, eps=EPS))
    for a, b in zip(got, want):
        assert all(torch.equal(u, v) for u, v in zip(a, b)) if isinstance(a, tuple) else torch.equal(a, b)
