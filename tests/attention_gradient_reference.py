"""Gradients of Stripe-Sort attention by their formulas in 64 bits, and how far a result in bf16 may be off them by norm.

Of every sum the squares of what its terms lose in bf16 are added up beside it: those of the probabilities P for dV, those of their gradients dS for dK and
dQ, and, where the bias' gradient G takes dS as one bf16 (grids above 32 x 32), those of dS for dQ and the tables once more.  Roundings of different terms are
independent, so the root of that, with the rounding of the result itself, is the norm of the error: thousands of roundings leave no room for a few per cent more
or less.  (A rounding to bf16 is off by 2^-8 of the value at most, 1.5e-3 at the root of the mean square.)"""
import math

import torch

BF = torch.bfloat16


def lost(x):
    """Squares of what x loses in bf16."""
    return (x.to(BF).double() - x) ** 2


def prefix(S, tile, r):
    return min(-(-S // tile), int(math.floor(r * -(-S // tile) + 1e-6)))


def scores(q, k, rel_h, rel_w, sigma, w, tile, r, scale, at):
    """Logits of the queries `at` of one head, -inf where the mask hides the key; and the relative positions of row and column."""
    S = q.shape[0]
    L = q[at] @ k.T * scale
    back = []
    for rel, cell in ((rel_h, sigma // w), (rel_w, sigma % w)):
        t = cell[at][:, None] - cell[None, :] + w - 1
        L = L + (q[at] @ rel.T).gather(1, t)
        back.append(t)
    tiles = torch.arange(S, device=q.device) // tile
    return L.masked_fill(~((tiles < prefix(S, tile, r))[None, :] | (tiles[None, :] == tiles[at][:, None])), -math.inf), back


def one_head(q, k, v, rel_h, rel_w, sigma, w, tile, r, do, out, scale, fine):
    """[S, d] in 64 bits; out: the result that delta is formed with.  -> gradients of q, k, v, rel_h, rel_w, and for each the squares of what its terms lose in bf16."""
    S = q.shape[0]
    some = max(1, (1 << 24) // S)
    grads = [torch.zeros_like(t) for t in (q, k, v, rel_h, rel_w)]
    loss = [torch.zeros_like(t) for t in grads]
    for first in range(0, S, some):
        at = torch.arange(first, min(first + some, S), device=q.device)
        L, back = scores(q, k, rel_h, rel_w, sigma, w, tile, r, scale, at)
        p = torch.softmax(L, 1)
        ds = p * (do[at] @ v.T - (do[at] * out[at]).sum(1, keepdim=True))
        lp, ls = lost(p), lost(ds)
        grads[0][at], loss[0][at] = ds @ k * scale, ls @ k ** 2 * scale ** 2
        grads[1] += ds.T @ q[at] * scale
        loss[1] += ls.T @ q[at] ** 2 * scale ** 2
        grads[2] += p.T @ do[at]
        loss[2] += lp.T @ do[at] ** 2
        for i, (rel, t) in enumerate(zip((rel_h, rel_w), back)):
            G, lg = (torch.zeros(at.numel(), 2 * w - 1, dtype=q.dtype, device=q.device).scatter_add_(1, t, m) for m in (ds, ls))
            grads[0][at] += G @ rel
            grads[3 + i] += G.T @ q[at]
            if not fine:
                loss[0][at] += lg @ rel ** 2
                loss[3 + i] += lg.T @ q[at] ** 2
    return grads, loss


def gradients(qkv, rel, sigma, w, tile, r, dout, out, out_rows=None, scale=None, heads=None):
    """Of a call: qkv [groups, S, 3, h, d], dout and out rows of h * d.  -> {(group, head): (dq, dk, dv)} of `heads` (all), drel_h, drel_w (all heads), and what
    they lose likewise."""
    groups, S, _, h, d = qkv.shape
    scale = d ** -0.5 if scale is None else scale
    fine = w <= 32
    tables = [t.double() for t in rel]
    single, table = {}, [[torch.zeros_like(t) for t in tables] for _ in range(2)]
    for g in range(groups):
        s = (sigma[g] if sigma.dim() == 2 else sigma).long()
        rows = torch.arange(g * S, g * S + S, device=qkv.device) if out_rows is None else out_rows.reshape(groups, S)[g].long()
        live = (rows >= 0)[:, None]
        for x in range(h):
            if heads is not None and (g, x) not in heads:
                continue
            q, k, v = (qkv[g, :, i, x].double() for i in range(3))
            do, o = (torch.where(live, t.reshape(-1, h, d)[rows.clamp(min=0), x].double(), 0.0) for t in (dout, out))
            q = torch.where(live, q, 0.0)
            grads, loss = one_head(q, k, v, *tables, s, w, tile, r, do, o, scale, fine)
            single[g, x] = (grads[:3], loss[:3])
            for i in range(2):
                table[0][i] += grads[3 + i]
                table[1][i] += loss[3 + i]
    return single, table


def off(got, ref, loss, what, factor=1.2, small=4e-4):
    """Norm of the error against the roundings': `factor` of their root and `small` of the reference's norm (bias entries in fp16, 2e-4 at the root of the mean square of a bias below
    one, and G in fp16 on grids, 2e-4 of itself; sums in 32 bits are far below).  -> the share of that"""
    got = got.double()
    assert torch.isfinite(got).all(), what
    norm = float(ref.norm())
    bound = factor * math.sqrt(float(lost(ref).sum() + loss.sum())) + small * norm + 1e-30
    err = float((got - ref).norm())
    print(f"[parity] {what}: off by {err / max(norm, 1e-300):.2e} of its norm, {err / bound:.3f} of the bound", flush=True)
    assert err <= bound, f"{what}: {err / bound:.3f} times the bound"
    return err / bound


def check(got, single, table, what, **kw):
    """got: (dqkv, drel_h, drel_w) of a call; every (group, head) by itself, so that none hides behind the others."""
    worst = 0.0
    dqkv, *drel = got
    for (g, x), (grads, loss) in single.items():
        for i, name in enumerate("qkv"):
            worst = max(worst, off(dqkv[g, :, i, x], grads[i], loss[i], f"d{name} of group {g}, head {x}, {what}", **kw))
    if table is not None:
        for i, name in enumerate(("drel_h", "drel_w")):
            worst = max(worst, off(drel[i], table[0][i], table[1][i], f"{name} {what}", **kw))
    return worst


def moves(L):
    """How often the reference of a query's running sums moves behind its first block of 32 keys: past a factor of 2^8 (L in natural units, keys in the order of the walk)."""
    n = -(-L.shape[1] // 32)
    L = torch.nn.functional.pad(L * math.log2(math.e), (0, 32 * n - L.shape[1]), value=-math.inf).view(L.shape[0], n, 32).amax(2)
    m, count = L[:, 0], torch.zeros(L.shape[0], dtype=torch.long, device=L.device)
    for i in range(1, n):
        move = L[:, i] > m + 8
        m, count = torch.where(move, L[:, i], m), count + move
    return count
