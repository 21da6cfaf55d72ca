"""The bounds of the step's differences (64 bits, no GPU): they refuse a gradient of zeros and one of the other sign."""
import pytest
import torch

import residual_differences as F
import residual_reference as R


@pytest.mark.parametrize("gate", ["features", "images"])
@pytest.mark.parametrize("second", [False, True])
def test_bounds_are_far_below_the_differences(gate, second):
    p, wx, wy = F.inputs(gate, second)
    assert all(torch.equal(t, t.float().double()) for t in p.values()) and torch.equal(p["x"], p["x"].to(torch.bfloat16).double())
    a = F.arguments(p, second)
    x_out = R.step(p["x"], p["o"], a["src"], a["post"], a["gate"], F.ALPHA, F.EPS)[0].to(torch.bfloat16).double()
    by = F.moves(p, F.gradients(p, x_out, wx, wy))
    for name in p:
        says, off, diff = F.allowed(p, x_out, name, by[name], wx, wy)
        print(name, says, diff, off)
        assert says > 4 * off and abs(says - diff) <= off, name
        for side in F.sides(p, name, by[name]):
            stored = side[name].to(torch.bfloat16 if name in ("x", "o") else torch.float32).double()
            assert torch.equal(stored, side[name])
