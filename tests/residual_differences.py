"""Differences of the step between two halves of a block along its own gradients: inputs whose moves are exact in the call's types, and how far a difference of the call may be from its gradient.

The loss is sum(wx * x_out) + sum(wy * y).  Every parameter moves along its gradient, so that the difference is the largest that a move of that length gives, many times what the call's
roundings can make of it: a gradient of zeros, or one of the other sign, is far outside."""
import torch

import residual_reference as R

B, N, NO, NY, D, ALPHA, EPS = 2, 8, 6, 7, 72, 0.9375, 1e-6
NAMES = ("x", "o", "gate", "post_g", "post_b", "pre_g", "pre_b")
SRC = torch.tensor([[3, -1, 0, 2, 1, 6, 5, 4], [-1, 1, 5, 9, 0, 3, 2, 4]], dtype=torch.int32)
DST = torch.tensor([1, -1, 0, 2, 7, 6, 4, 3], dtype=torch.int32)


def inputs(gate, second):
    """x and o are sixteenths of up to 64 (they and two sixteenths more are exact in bf16), wx and wy bf16 values; ``second``: with the second LayerNorm"""
    gen = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    sixteenths = lambda *s: (n(*s) * 16).round().clamp(-64, 64).double() / 16  # noqa: E731
    p = {"x": sixteenths(B, N, D), "o": sixteenths(B, NO, D), "gate": (0.7 + 0.3 * n(*((B, D) if gate == "images" else (D,)))).double(),
         "post_g": (1 + 0.2 * n(D)).double(), "post_b": (0.2 * n(D)).double()}
    if second:
        p |= {"pre_g": (1 + 0.2 * n(D)).double(), "pre_b": (0.2 * n(D)).double()}
    w = lambda *s: n(*s).to(torch.bfloat16).double()  # noqa: E731
    return p, w(B, N, D), w(B, NY, D) if second else None


def arguments(p, second):
    return dict(src=SRC, post=(p["post_g"], p["post_b"]), gate=p["gate"], alpha=ALPHA, pre=(p["pre_g"], p["pre_b"]) if second else None, dst=DST if second else None, eps=EPS)


def gradients(p, x_out, wx, wy):
    """{name: (gradient in 64 bits, what fp32 and the rounding of what is stored may be off)}"""
    a = arguments(p, wy is not None)
    form = (x_out, p["o"], a["src"], a["post"], a["gate"], a["alpha"], a["pre"], a["dst"], EPS, wy, wx)
    got, err = R.step_gradients(*form), R.step_gradient_errors(*form)
    return {n: (got["d" + n], err["d" + n] + got["d" + n].abs() * (R.BF if n in ("x", "o") else R.U)) for n in p}


def loss(p, wx, wy):
    """-> the loss in 64 bits, and how far that of the call may be off: the stream and y are rounded to bf16 once, half a step each, the stream's rounding goes through the second LayerNorm
    (to first order; a tenth more bounds the rest, 2^-8 of it), and what fp32 is off."""
    a = arguments(p, wy is not None)
    out, e = R.step(p["x"], p["o"], a["src"], a["post"], a["gate"], ALPHA, EPS)
    there = R.rows_of(a["src"], p["o"], B)[1]
    e = torch.where(there, e + R.BF * out.abs(), 0.0)
    total, off = (out * wx).sum(), (wx.abs() * e).sum()
    if wy is not None:
        h, rstd = R.layer_norm(out, EPS)
        mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
        y = h * a["pre"][0] + a["pre"][1]
        ey = a["pre"][0].abs() * (rstd * (e + mean(e) + h.abs() * mean(h.abs() * e)) + R.layer_norm_error(out, EPS)) + 2 * R.U * (y.abs() + a["pre"][1].abs()) + R.BF * y.abs()
        g, named = R.rows_of(DST, wy, B)
        g = torch.where(named, g, 0.0)
        total, off = total + (y * g).sum(), off + (g.abs() * ey).sum()
    return total, 1.1 * off


def moves(p, grads):
    """{name: by}: of x and o two sixteenths in their gradient's direction, of the others along it, a quarter long each entry on average (fp32, so that the call has the same)"""
    by = {}
    for n, t in p.items():
        g = grads[n][0]
        by[n] = torch.sign(g) / 8 if n in ("x", "o") else (g * (0.25 * g.numel() ** 0.5 / g.norm())).float().double()
        if n not in ("x", "o"):
            by[n] = (t.float() + by[n].float()).double() - t           # (what the sum in fp32 moves by)
    return by


def sides(p, name, by):
    """The parameters with one moved there and back; values that fp32 has"""
    there, back = p[name] + by, p[name] - by
    if name not in ("x", "o"):
        back = back.float().double()
    return {**p, name: there}, {**p, name: back}


def allowed(p, x_out, name, by, wx, wy):
    """-> what the gradient says of the difference of both sides, and how far the call's difference may be from it: roundings of both, of the gradient, and the curvature, which is what the
    difference in 64 bits is off by itself."""
    one, two = sides(p, name, by)
    whole = one[name] - two[name]
    g, err = gradients(p, x_out, wx, wy)[name]
    says = (g * whole).sum()
    (l1, e1), (l2, e2) = loss(one, wx, wy), loss(two, wx, wy)
    return float(says), float(e1 + e2 + (l1 - l2 - says).abs() + (err * whole.abs()).sum()), float(l1 - l2)
