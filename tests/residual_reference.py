"""The step between two halves of a block and rows in 8 bits, in 64 bits on the CPU, and what 32-bit arithmetic may add to their rounding."""
import numpy as np
import torch

U = 2.0 ** -24                # half a step of fp32, relative
BF = 2.0 ** -8                # of bf16


def layer_norm(v, eps):
    """rows -> (normalised rows, one over their deviation)"""
    v = v - v.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)
    return v * rstd, rstd


def layer_norm_error(v, eps):
    """How far normalised rows may be off in fp32: sums of D terms are 32 in a lane and a tree of six, 38 roundings, and a mean is one more; the mean's error goes
    through the deviation (once into the row, and, times h, into its variance, whose own 40 roundings count half)."""
    h, rstd = layer_norm(v, eps)
    return 45 * U * v.abs().mean(-1, keepdim=True) * rstd * (1 + h.abs()) + 30 * U * h.abs()


def rows_of(which, values, B):
    """values [B,rows,D] by a map [N] or [B,N] -> ([B,N,D], [B,N,1] whether there is one)"""
    m = which.expand(B, -1).long()
    there = (m >= 0) & (m < values.shape[1])
    return torch.gather(values, 1, torch.where(there, m, 0)[..., None].expand(-1, -1, values.shape[2])), there[..., None]


def own_order(B, N):
    return torch.arange(N)[None].expand(B, -1)


def step(x, o, src, post, gate, alpha, eps):
    """The stream behind the step in 64 bits, and what fp32 may be off before it is rounded."""
    B, N, D = x.shape
    if o is None:
        return x, torch.zeros_like(x)
    n, there = rows_of(own_order(B, N) if src is None else src, o, B)
    err = torch.zeros_like(n)
    if post is not None:
        h = layer_norm(n, eps)[0]
        err = layer_norm_error(n, eps) * post[0].abs() + U * (h * post[0]).abs()
        n = h * post[0] + post[1]
        err = err + U * n.abs()
    if gate is not None:
        g = gate[:, None] if gate.dim() == 2 else gate
        err = err * g.abs() + U * (n * g).abs()
        n = n * g
    new = alpha * x + n
    return torch.where(there, new, x), torch.where(there, err + U * new.abs() + U * (alpha * x).abs(), 0.0)


def step_gradients(x_out, o, src, post, gate, alpha, pre, dst, eps, dy, dx_out):
    """By differentiation of the formulas in 64 bits: {name: gradient}.  x_out: the stream behind the step, as it was stored."""
    B, N, D = x_out.shape
    leaf = lambda t: None if t is None else t.detach().clone().requires_grad_()  # noqa: E731
    o, gate, before = leaf(o), leaf(gate), torch.zeros_like(x_out, requires_grad=True)
    post, pre = (None if p is None else (leaf(p[0]), leaf(p[1])) for p in (post, pre))
    up = torch.zeros_like(x_out) if dx_out is None else dx_out.clone()
    got = {}
    if pre is not None:
        x = leaf(x_out)
        g, there = rows_of(own_order(B, N) if dst is None else dst, dy, B)
        (layer_norm(x, eps)[0] * pre[0] + pre[1]).backward(torch.where(there, g, 0.0))
        up = up + x.grad
        got |= {"dpre_g": pre[0].grad, "dpre_b": pre[1].grad}
    step(before, o, src, post, gate, alpha, eps)[0].backward(up)
    got["dx"] = before.grad
    for name, t in (("do", o), ("dgate", gate), *((("dpost_g", post[0]), ("dpost_b", post[1])) if post else ())):
        if t is not None:
            got[name] = torch.zeros_like(t) if t.grad is None else t.grad
    return got


def step_gradient_errors(x_out, o, src, post, gate, alpha, pre, dst, eps, dy, dx_out):
    """What fp32 may be off in each of them: every value is formed of a few terms, and of two sums over a row (38 roundings each) of terms that have the rows' own errors;
    100 roundings of the terms' magnitudes, times 1 + (a row's mean magnitude over its deviation, which normalised rows are that much less exact by), bound all of
    it.  Sums over rows add at most 64 more: 64 rows a wave here and in the tests' sizes, 4 waves, 16 of 512 workgroups, a tree of five."""
    B, N, D = x_out.shape
    mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
    G = torch.zeros_like(x_out) if dx_out is None else dx_out.abs()
    got, worse = {}, torch.ones(B, N, 1, dtype=torch.float64)

    def back(g, h, rstd, loss):               # magnitudes through a LayerNorm's gradient
        return rstd * (g + mean(g) + h * mean(g * h) + (h + 1) * mean(g * (h + 1)) * loss * U * 50)

    if pre is not None:
        g, there = rows_of(own_order(B, N) if dst is None else dst, dy.abs(), B)
        g = torch.where(there, g, 0.0)
        h, rstd = layer_norm(x_out, eps)
        loss = torch.where(there, mean(x_out.abs()) * rstd, 0.0)
        got |= {"dpre_g": (164 * U * (1 + loss) * g * (h.abs() + 1)).sum((0, 1)), "dpre_b": (164 * U * g).sum((0, 1))}
        worse = worse + loss
        G = G + torch.where(there, back(g * pre[0].abs(), h.abs(), rstd, loss), 0.0)
    if o is None:
        got["dx"] = 100 * U * worse * G
        return got
    m = (own_order(B, N) if src is None else src).expand(B, -1).long()
    n, there = rows_of(m, o, B)
    got["dx"] = 100 * U * worse * torch.where(there, abs(alpha) * G, G)
    G = torch.where(there, G, 0.0)
    dn, h, rstd, loss = G, n.abs(), None, torch.zeros_like(worse)
    if gate is not None:
        dn = dn * (gate[:, None] if gate.dim() == 2 else gate).abs()
    if post is not None:
        h, rstd = layer_norm(n, eps)
        h, loss = h.abs(), mean(n.abs()) * rstd
        worse = worse + loss
        got |= {"dpost_g": (164 * U * worse * dn * (h + 1)).sum((0, 1)), "dpost_b": (164 * U * worse * dn).sum((0, 1))}
        times = h * post[0].abs() + post[1].abs() + post[0].abs()
        dn = back(dn * post[0].abs(), h, rstd, loss)
    else:
        times = n.abs()
    if gate is not None:
        d = (164 * U * worse * G * times).sum(1)
        got["dgate"] = d if gate.dim() == 2 else d.sum(0)
    do = torch.zeros_like(o)
    b, t = torch.nonzero(there[..., 0], as_tuple=True)
    do[b, m[b, t]] = (100 * U * worse * dn)[b, t]
    got["do"] = do
    return got


def quantised(x):
    """bf16 rows (fp32 or fp64 arrays of such values) -> (codes int8, scales fp32).  x * 127 is exact in 64 bits, and a quotient by a bf16 number is a tie or 7e-6 from one."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(axis=-1)
    safe = np.where(top > 0, top, 1.0)
    scales = np.maximum(top.astype(np.float32) / np.float32(127), np.float32(2.0 ** -126))
    step = np.maximum(safe / 127, 2.0 ** -126)
    codes = np.rint(np.where((step > 2.0 ** -126)[..., None], x * 127 / safe[..., None], x / 2.0 ** -126))
    return codes.astype(np.int8), scales.astype(np.float32)
