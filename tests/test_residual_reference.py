"""The 64-bit gradients of the step between two halves of a block against differences of its formulas."""
import pytest
import torch

import residual_reference as R

B, N, D = 2, 5, 8


@pytest.mark.parametrize("post,gate,pre,alpha", [(True, "images", True, 0.75), (False, "features", True, 1.0), (True, "none", False, -0.5), (False, "none", True, 0.0)])
def test_gradients_against_differences(post, gate, pre, alpha):
    gen = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    x, o, src, dst = n(B, N, D), n(B, 4, D), torch.tensor([[3, -1, 0, 2, 1], [-1, 1, -1, 9, 0]]), torch.tensor([1, -1, 0, 2, 7])
    p = {"x": x, "o": o}
    if post:
        p |= {"post_g": 1 + n(D), "post_b": n(D)}
    if gate != "none":
        p["gate"] = n(B, D) if gate == "images" else n(D)
    if pre:
        p |= {"pre_g": 1 + n(D), "pre_b": n(D)}
    wx, wy = n(B, N, D), n(B, 3, D)

    def loss(p):
        out = R.step(p["x"], p["o"], src, (p["post_g"], p["post_b"]) if post else None, p.get("gate"), alpha, 1e-6)[0]
        total = (out * wx).sum()
        if pre:
            y = R.layer_norm(out, 1e-6)[0] * p["pre_g"] + p["pre_b"]
            g, there = R.rows_of(dst, wy, B)
            total = total + torch.where(there, y * g, 0.0).sum()
        return total

    out = R.step(x, o, src, (p["post_g"], p["post_b"]) if post else None, p.get("gate"), alpha, 1e-6)[0]
    got = R.step_gradients(out, o, src, (p["post_g"], p["post_b"]) if post else None, p.get("gate"), alpha, (p["pre_g"], p["pre_b"]) if pre else None, dst, 1e-6,
                           wy if pre else None, wx)
    assert set(got) == {"d" + k for k in p}
    for name, t in p.items():
        d, h = n(*t.shape), 1e-5
        diff = (loss({**p, name: t + h * d}) - loss({**p, name: t - h * d})) / (2 * h)
        # a central difference is off by h^2 times the third derivative (1e-10 of sizes near 100) and by 64-bit rounding over h (1e-14 / 1e-5 of them)
        assert abs(float(diff - (got["d" + name] * d).sum())) <= 1e-6, name


def test_codes():
    codes, scales = R.quantised([[127.0, 63.5, -64.5, 0.25], [0, 0, 0, 0], [2.0 ** -130, 0, 0, 0]])
    assert codes.tolist() == [[127, 64, -64, 0], [0, 0, 0, 0], [0, 0, 0, 0]] and scales[0] == 1.0 and scales[1] == scales[2] == 2.0 ** -126
