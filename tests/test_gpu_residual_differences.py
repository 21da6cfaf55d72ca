"""Gradients of the step against differences of the step's own call, along them: every gradient, with and without a second LayerNorm."""
import pytest
import torch

import residual_differences as F
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _device(p, second):
    a = F.arguments({n: t.float().to(DEV) for n, t in p.items()}, second)
    stream = {n: p[n].to(torch.bfloat16).to(DEV) for n in ("x", "o")}
    return stream["x"], stream["o"], {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in a.items()}


@pytest.mark.parametrize("gate", ["features", "images"])
@pytest.mark.parametrize("second", [False, True])
def test_gradients(gate, second):
    p, wx, wy = F.inputs(gate, second)

    def call(p):
        x, o, a = _device(p, second)
        return B.ssam_residual_norm(x, o, **a, Ny=F.NY)

    x_out, _ = call(p)
    _, o, a = _device(p, second)
    dx, do, dgate, dpost, dpre = B.ssam_residual_norm_backward(x_out, o, **a, dy=wy.to(torch.bfloat16).to(DEV) if second else None, dx_out=wx.to(torch.bfloat16).to(DEV))
    got = dict(zip(F.NAMES, (dx, do, dgate, *dpost, *(dpre or ()))))
    stored = x_out.double().cpu()
    by = F.moves(p, F.gradients(p, stored, wx, wy))
    assert set(got) == set(p)
    for name in p:
        losses = []
        for side in F.sides(p, name, by[name]):
            out, y = call(side)
            total = (out.double().cpu() * wx).sum()
            if second:
                g, named = F.R.rows_of(F.DST, y.double().cpu(), F.B)
                w = F.R.rows_of(F.DST, wy, F.B)[0]
                total = total + torch.where(named, g * w, 0.0).sum()
            losses.append(float(total))
        one, two = F.sides(p, name, by[name])
        says = float((got[name].double().cpu() * (one[name] - two[name])).sum())
        _, off, _ = F.allowed(p, stored, name, by[name], wx, wy)
        announce("differences", gate, second, name, says, losses[0] - losses[1], off)
        assert says > 4 * off and abs(losses[0] - losses[1] - says) <= off, name
