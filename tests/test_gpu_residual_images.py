"""Gradients of the step with a gate of every image, for numbers of images that do not divide the CUs, against formulas in 64 bits."""
import pytest
import torch

import residual_reference as R
from helpers import announce
from paper_2605_17633_amd import binding as B
from test_gpu_residual import DEV, EPS, STEP, _dev, _double, _inputs, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("images,N,D,post", [(5, 700, 520, True), (7, 500, 1280, True), (6, 300, 2048, True), (7, 90, 1152, False), (129, 40, 144, True), (129, 20, 1024, True), (255, 12, 256, False)])
def test_images(images, N, D, post):
    case = (images, N, max(1, N - N // 3), max(1, N // 2), D, post, "images", True, 0.9375, "each")
    announce("residual_norm_backward", case)
    s = _inputs(case, 11)
    d, r = _dev(s), _double(s)
    need = B.ssam_residual_norm_backward_workspace_bytes(images, N, D, images)
    room = torch.full((need + 512,), 77, dtype=torch.uint8, device=DEV)
    args = {k: d[k] for k in (*STEP, "dy", "dx_out")}
    runs = [B.ssam_residual_norm_backward(d["x"], **args, eps=EPS, workspace=room[256:256 + need]) for _ in range(2)]
    assert bool((room[:256] == 77).all()) and bool((room[256 + need:] == 77).all())
    flat = lambda g: (g[0], g[1], g[2], *(g[3] or ()), *g[4])  # noqa: E731
    assert all(torch.equal(a, b) for a, b in zip(*map(flat, runs)))
    form = (r["x"], r["o"], r["src"], r["post"], r["gate"], r["alpha"], r["pre"], r["dst"], EPS, r["dy"], r["dx_out"])
    want, err = R.step_gradients(*form), R.step_gradient_errors(*form)
    for name, t in zip(("dx", "do", "dgate", *(("dpost_g", "dpost_b") if post else ()), "dpre_g", "dpre_b"), flat(runs[0])):
        _within(t, want[name], err[name], name, step=R.BF if name in ("dx", "do") else R.U)
