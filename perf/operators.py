"""What a training step adds to the encoder block, as calls of the library and in plain form: how fast each is, and how far off.

A case is a dict of plain values.  Its ``path`` says which operator it stands for:

  attention   gradients of Stripe-Sort attention (``ssam_sparse_attention_backward``): from the packed q/k/v tensor, the
              forward's result and its gradient to the gradients of q, k, v and of the two relative-position tables
  layernorm   gradients of the LayerNorm of gathered tokens (``ssam_ln_gather_backward``): into the gradient of the residual
              stream, which they are added to or written over, and of the LayerNorm's own weights
  checkpoint  an activation kept in 8 bits between the passes (``ssam_checkpoint_store``, ``ssam_checkpoint_restore``)
  gelu        the MLP's activation with its argument kept in 8 bits: forward (``ssam_gelu_checkpoint``) and backward
              (``ssam_gelu_backward``), which gives the activation again for the gradient of fc2's weights

The attention density is that of the A-shape mask: every query has the first floor(density * T) of the T tiles of keys, and
its own.  ``order`` is the scan order: ``position`` (one table for all groups) or ``content`` (a table for every group).
"""
import math

import torch

own = False

DEV = "cuda"
BF = torch.bfloat16
STRIPE = 4            # G of the stripe interleave
LN_EPS = 1e-6
COLS = 64             # columns that share a scale in 8 bits


def listed():
    return [
        # one small grid, dense: the least that a program tries first, bound by latency
        dict(name="attention_global_28x28_b1", path="attention", batch=1, grid=28, window=0, heads=12, dim=64, density=1.0, order="position"),
        # the windows of one 1024 x 1024 image, base width: the padding slots of the border windows have no output
        dict(name="attention_windows_b1", path="attention", batch=1, grid=64, window=14, heads=12, dim=64, density=0.4, order="position"),
        # windows of a training batch at the huge width, ordered by content: a table for every window
        dict(name="attention_windows_content_b4", path="attention", batch=4, grid=64, window=14, heads=16, dim=80, density=0.5, order="content"),
        # a global block of one image, large width
        dict(name="attention_global_b1", path="attention", batch=1, grid=64, window=0, heads=16, dim=64, density=0.4, order="position"),
        # a grid that is not a power of two (800 pixels), ordered by content
        dict(name="attention_global_50x50_b2", path="attention", batch=2, grid=50, window=0, heads=12, dim=64, density=0.5, order="content"),
        # a global block of a training batch at the huge width: the largest
        dict(name="attention_global_b4", path="attention", batch=4, grid=64, window=0, heads=16, dim=80, density=0.4, order="position"),
        # LN2 of the kept tokens of one small image: latency
        dict(name="layernorm_kept_b1", path="layernorm", batch=1, grid=28, width=768, rows="kept", density=0.4, accumulate=True),
        # LN1 of a batch in window order: padding slots among the rows; its gradient joins the residual stream's
        dict(name="layernorm_windows_b8", path="layernorm", batch=8, grid=64, width=1280, rows="windows", density=1.0, accumulate=True),
        # a block's input kept for the backward pass
        dict(name="checkpoint_b8", path="checkpoint", rows=32768, width=1280),
        # a stage of a hierarchical encoder: width that is no multiple of the 64 columns of a scale
        dict(name="checkpoint_144", path="checkpoint", rows=4900, width=144),
        # the hidden layer of the routed MLP: a stage of a hierarchical encoder, and a batch at the huge width
        dict(name="gelu_576", path="gelu", rows=612, width=576),
        dict(name="gelu_5120_b8", path="gelu", rows=13104, width=5120),
    ]


def draw(rng):
    """One more case of the same ranges: windows of 4 x 4 to 14 x 14 and grids up to 72 x 72, all head sizes, orders and densities;
    rows of 8 to 2048 features from one token to 32768; 8-bit rows up to 5120 wide."""
    between = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        path = rng.choice(["attention", "attention", "attention", "layernorm", "checkpoint", "gelu"])
        if path == "attention":
            window = rng.choice([0, 0, 14, between(4, 14)])
            case = dict(path=path, batch=between(1, 6), grid=between(8, 72) if window == 0 else between(max(window, 8), 72), window=window,
                        heads=rng.choice([1, 3, 8, 12, 16]), dim=rng.choice([16, 32, 64, 64, 80, 80]),
                        density=rng.choice([0.2, 0.3, 0.4, 0.5, 0.6, 1.0]), order=rng.choice(["position", "content"]))
        elif path == "layernorm":
            case = dict(path=path, batch=between(1, 8), grid=between(1, 64), width=rng.choice([768, 1024, 1280, 8 * between(1, 256)]),
                        rows=rng.choice(["kept", "windows"]), density=rng.choice([0.1, 0.3, 0.4, 0.7, 1.0]), accumulate=rng.random() < 0.5)
        else:
            case = dict(path=path, rows=between(1, 32768), width=rng.choice([768, 1280, 4096, 5120, 8 * between(1, 640)]))
        if _cost(case) <= _MOST[path]:
            return case


# ------------------------------------------------------------------ sizes
def _attention_sizes(case):
    """-> groups, side of a group, tokens of a group, key tile, tiles in front"""
    w = case["window"] or case["grid"]
    groups = case["batch"] * (-(-case["grid"] // w)) ** 2
    tile = 32 if case["window"] else 128
    S = w * w
    return groups, w, S, tile, min(-(-S // tile), int(math.floor(case["density"] * -(-S // tile) + 1e-6)))


def _pairs(case):
    """Pairs of a query and a key that the mask lets see each other, in one group and head."""
    groups, w, S, tile, ahead = _attention_sizes(case)
    front = min(S, ahead * tile)
    return S * front + sum(min(tile, S - t) ** 2 for t in range(front, S, tile))


def _kept(case):
    n = case["grid"] ** 2
    return max(1, min(n, int(math.floor(case["density"] * n + 1e-6))))


def work(case):
    """Bytes (inputs and outputs once) and flops of one pass."""
    if case["path"] == "attention":
        groups, w, S, tile, ahead = _attention_sizes(case)
        features = case["heads"] * case["dim"]
        tokens = case["batch"] * case["grid"] ** 2                # rows of the forward's result and of its gradient
        tables = 2 * (2 * w - 1) * case["dim"]
        sigma = 4.0 * S * (groups if case["order"] == "content" else 1)
        # five products over the pairs (scores, the gradient of the probabilities, and the gradients of q, k and v); a bias entry
        # of a query and a row or column is a product of d, and so are the two that its gradient goes into
        return {"bytes": 2.0 * features * (6 * groups * S + 2 * tokens) + 2.0 * 2 * tables + sigma + (4.0 * groups * S if case["window"] else 0),
                "flops": (10.0 * _pairs(case) + 3 * 2.0 * S * 2 * w) * case["dim"] * case["heads"] * groups}
    if case["path"] == "layernorm":
        n, D = case["grid"] ** 2, case["width"]
        named = case["batch"] * (_kept(case) if case["rows"] == "kept" else n)
        return {"bytes": 2.0 * named * D * (4 if case["accumulate"] else 3) + 12.0 * D, "flops": 14.0 * named * D}
    rows, D = case["rows"], case["width"]
    if case["path"] == "checkpoint":                              # read, codes written and read, written
        return {"bytes": rows * (2.0 * D + 2 * (D + 4.0 * -(-D // COLS)) + 2 * D), "flops": 4.0 * rows * D}
    return {"bytes": rows * (4.0 * D + 2 * (D + 4.0 * -(-D // COLS)) + 6 * D), "flops": 40.0 * rows * D}


def _cost(case):
    return work(case)["flops"]


#: no drawn case is more work than the largest listed one of its path
_MOST = {}
for _c in listed():
    _MOST[_c["path"]] = max(_MOST.get(_c["path"], 0.0), _cost(_c))
_MOST["checkpoint"] = max(_MOST["checkpoint"], 4.0 * 32768 * 1280)


# ------------------------------------------------------------------ inputs
def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(dtype)


def _z_order(w):
    """Cells of a w x w grid along the Z-order curve: columns are the even bits of a cell's code, rows the odd ones."""
    i = torch.arange(w * w, device=DEV)
    row, col = i // w, i % w
    code = sum((((col >> b) & 1) << (2 * b)) | (((row >> b) & 1) << (2 * b + 1)) for b in range(8))
    return torch.argsort(code)


def _stripes(order):
    """The stripe interleave of an order [..., S]: every STRIPE-th cell, then the next ones.  Sizes that it does not divide stay as they are."""
    S = order.shape[-1]
    if S % STRIPE:
        return order.contiguous()
    return order.view(*order.shape[:-1], S // STRIPE, STRIPE).transpose(-1, -2).reshape(order.shape)


def _window_cells(g, w, window):
    """[groups of one image, w*w]: the token at every cell of every group, -1 where the grid has none."""
    side = -(-g // w) if window else 1
    at = torch.arange(w, device=DEV)
    row = torch.arange(side, device=DEV)[:, None] * w + at                       # [side, w]
    token = row[:, None, :, None] * g + row[None, :, None, :]                    # [side, side, w, w]
    inside = (row[:, None, :, None] < g) & (row[None, :, None, :] < g)
    return torch.where(inside, token, -1).reshape(side * side, w * w)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return {"case": case, **_PREPARE[case["path"]](case, gen)}


def _prepare_attention(case, gen):
    groups, w, S, tile, ahead = _attention_sizes(case)
    h, d, batch, n = case["heads"], case["dim"], case["batch"], case["grid"] ** 2
    cells = _window_cells(case["grid"], w, case["window"]).repeat(batch, 1)      # [groups, S]
    if case["order"] == "content":                                                # by score, the highest first; cells without a token last
        score = torch.where(cells >= 0, torch.rand(groups, S, generator=gen, device=DEV), -1.0)
        sigma = _stripes(torch.argsort(score, dim=1, descending=True, stable=True))
        token = torch.gather(cells, 1, sigma)
    else:
        sigma = _stripes(_z_order(w))
        token = cells[:, sigma]
    image = torch.arange(groups, device=DEV)[:, None] // (groups // batch)
    rows = torch.where(token >= 0, token + image * n, -1)
    s = {"sigma": sigma.to(torch.int32).contiguous(), "out_rows": rows.to(torch.int32).contiguous() if case["window"] else None, "w": w,
         "qkv": _normal(gen, groups, S, 3, h, d, std=0.7, dtype=BF),
         "rel": (_normal(gen, 2 * w - 1, d, std=0.1, dtype=BF), _normal(gen, 2 * w - 1, d, std=0.1, dtype=BF)),
         "dout": _normal(gen, batch * n, h * d, std=0.02, dtype=BF)}
    out = torch.zeros(batch * n, h, d, dtype=BF, device=DEV)
    to = rows.reshape(-1)
    some = max(1, (1 << 28) // (h * S * S))                                       # groups at a time
    for g in range(0, groups, some):
        part = slice(g, min(g + some, groups))
        q, k, v = _heads_first(s["qkv"][part].float())
        p = _probabilities(q, k, *s["rel"], s["sigma"][part] if s["sigma"].dim() == 2 else s["sigma"], w, tile, ahead, q.shape[0] // h)[0]
        o = (p @ v).view(-1, h, S, d).transpose(1, 2).reshape(-1, h, d).to(BF)
        at = to[part.start * S:part.stop * S]
        out[at[at >= 0]] = o[at >= 0]
        del p
    s["out"] = out.view(batch * n, h * d)
    if not case["window"]:
        s["out"], s["dout"] = s["out"].view(groups, S, -1), s["dout"].view(groups, S, -1)
        s["out"] = torch.gather(s["out"], 1, rows.sub(image * n)[:, :, None].expand(-1, -1, h * d)).contiguous()      # scan order
    return s


def _prepare_layernorm(case, gen):
    batch, g, D = case["batch"], case["grid"], case["width"]
    n = g * g
    if case["rows"] == "kept":
        k = _kept(case)
        idx = torch.rand(batch, n, generator=gen, device=DEV).argsort(dim=1)[:, :k].sort(dim=1)[0].to(torch.int32)
    else:
        w = min(14, g)
        idx = _window_cells(g, w, True)[:, _stripes(_z_order(w))].reshape(1, -1).to(torch.int32)
    return {"x": _normal(gen, batch, n, D, dtype=BF) + _normal(gen, 1, 1, D, std=0.5, dtype=BF), "idx": idx.contiguous(),
            "gamma": 1 + _normal(gen, D, std=0.1), "dy": _normal(gen, batch, idx.shape[1], D, std=0.02, dtype=BF),
            "g0": _normal(gen, batch, n, D, std=0.02, dtype=BF)}


def _prepare_rows(case, gen):
    # activations: a scale of their own for every feature, as trained networks have, a few of them much larger
    spread = torch.exp(_normal(gen, case["width"], std=0.5))
    x = (_normal(gen, case["rows"], case["width"]) * spread).to(BF)
    return {"x": x, "da": _normal(gen, case["rows"], case["width"], std=0.02, dtype=BF) if case["path"] == "gelu" else None}


# ------------------------------------------------------------------ passes
def run(state):
    return _RUN[state["case"]["path"]](state, state["case"])


def _heads_first(qkv):
    """[groups, S, 3, h, d] -> q, k, v of [groups * h, S, d]"""
    t = qkv.permute(2, 0, 3, 1, 4)
    return [x.reshape(-1, *x.shape[2:]) for x in t]


def _one_hot(at, w):
    """[..., S] -> [..., S, w]"""
    return (at[..., None] == torch.arange(w, device=at.device)).float()


def _probabilities(q, k, rel_h, rel_w, sigma, w, tile, ahead, groups):
    """-> P [groups * h, S, S], and what the gradients of the bias need: per table, U[i, y] = q_i . rel[at_i - y + w - 1] comes from the
    positions t = at_i - y + w - 1 of a query and an entry y."""
    h, S = q.shape[0] // groups, q.shape[1]
    sigma = sigma.long().expand(groups, S)
    logits = (q @ k.transpose(1, 2)) * q.shape[2] ** -0.5
    back = []
    for table, at in ((rel_h, sigma // w), (rel_w, sigma % w)):
        t = at[:, :, None] - torch.arange(w, device=q.device) + (w - 1)           # [groups, S, w]
        t = t.repeat_interleave(h, 0)
        hot = _one_hot(at, w).repeat_interleave(h, 0)
        logits += torch.gather(q @ table.float().t(), 2, t) @ hot.transpose(1, 2)
        back.append((table, t, hot))
    i = torch.arange(S, device=q.device) // tile
    logits = logits.masked_fill((i[None, :] >= ahead) & (i[None, :] != i[:, None]), -math.inf)
    p = torch.exp(logits - logits.amax(2, keepdim=True))
    return p / p.sum(2, keepdim=True), back


def _run_attention(s, case):
    groups, w, S, tile, ahead = _attention_sizes(case)
    if own:
        from paper_2605_17633_amd import binding as B
        dqkv, drel_h, drel_w = B.ssam_sparse_attention_backward(s["qkv"], *s["rel"], s["sigma"], w, tile, case["density"], s["out"], s["dout"],
                                                                out_rows=s["out_rows"])
        return {"dq": dqkv[:, :, 0], "dk": dqkv[:, :, 1], "dv": dqkv[:, :, 2], "drel_h": drel_h, "drel_w": drel_w}
    h, d = case["heads"], case["dim"]
    q, k, v = _heads_first(s["qkv"].float())
    p, back = _probabilities(q, k, *s["rel"], s["sigma"], w, tile, ahead, groups)
    do = s["dout"].reshape(-1, h, d).float()
    if s["out_rows"] is not None:
        rows = s["out_rows"].reshape(-1).long()
        do = do[rows.clamp(min=0)] * (rows >= 0)[:, None, None]
    do = do.view(groups, S, h, d).transpose(1, 2).reshape(-1, S, d)
    dv = p.transpose(1, 2) @ do
    ds = do @ v.transpose(1, 2)
    ds = p * (ds - (p * ds).sum(2, keepdim=True))
    dq = (ds @ k) * d ** -0.5
    dk = (ds.transpose(1, 2) @ q) * d ** -0.5
    drel = []
    for table, t, hot in back:
        du = torch.zeros(*t.shape[:2], 2 * w - 1, device=DEV).scatter_(2, t, ds @ hot)
        dq += du @ table.float()
        drel.append((du.transpose(1, 2) @ q).sum(0).to(BF))
    dq, dk, dv = (x.view(groups, h, S, d).transpose(1, 2).to(BF).contiguous() for x in (dq, dk, dv))
    return {"dq": dq, "dk": dk, "dv": dv, "drel_h": drel[0], "drel_w": drel[1]}


def _run_layernorm(s, case):
    x, idx, gamma, dy = s["x"], s["idx"], s["gamma"], s["dy"]
    dx = s["g0"].clone()                                          # the gradient of the stream so far, which the call updates in place
    if own:
        from paper_2605_17633_amd import binding as B
        dx, dgamma, dbeta = B.ssam_ln_gather_backward(x, idx, 0 if idx.shape[0] == 1 else idx.shape[1], gamma, LN_EPS, dy, dx=dx,
                                                      accumulate=case["accumulate"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    b, p = torch.nonzero(idx.expand(x.shape[0], -1) >= 0, as_tuple=True)
    src = idx.expand(x.shape[0], -1)[b, p].long()
    v, g = x[b, src].float(), dy[b, p].float()
    v = v - v.mean(1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + LN_EPS)
    v = v * rstd
    dgamma, dbeta = (g * v).sum(0), g.sum(0)
    g = g * gamma
    g = (g - g.mean(1, keepdim=True) - v * (g * v).mean(1, keepdim=True)) * rstd
    dx[b, src] = ((dx[b, src].float() if case["accumulate"] else 0) + g).to(BF)
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _codes(x):
    """Whole numbers of -127 to 127 and the scale of every COLS columns: x is about codes * scale."""
    rows, D = x.shape
    blocks = torch.nn.functional.pad(x.float(), (0, -D % COLS)).view(rows, -1, COLS)
    top = blocks.abs().amax(2, keepdim=True)
    scale = (top / 127).clamp(min=2.0 ** -126)
    codes = torch.round(blocks * torch.where(top > 0, (127 / top).clamp(max=2.0 ** 126), 0.0))
    return codes, scale


def _values(codes, scale, D):
    return (codes * scale).flatten(1)[:, :D]


def _run_checkpoint(s, case):
    if own:
        from paper_2605_17633_amd import binding as B
        codes, scales = B.ssam_checkpoint_store(s["x"])
        return {"x": B.ssam_checkpoint_restore(codes, scales)}
    return {"x": _values(*_codes(s["x"]), case["width"]).to(BF)}


def _run_gelu(s, case):
    if own:
        from paper_2605_17633_amd import binding as B
        a, codes, scales = B.ssam_gelu_checkpoint(s["x"])
        dh, again = B.ssam_gelu_backward(codes, scales, s["da"])
        return {"a": a, "dh": dh, "a_again": again}
    x = s["x"].float()
    t = _values(*_codes(s["x"]), case["width"])
    cdf = 0.5 * torch.erfc(t * -math.sqrt(0.5))
    slope = cdf + t * torch.exp(t * t * -0.5) * (1 / math.sqrt(2 * math.pi))
    return {"a": (0.5 * x * torch.erfc(x * -math.sqrt(0.5))).to(BF), "dh": (s["da"].float() * slope).to(BF), "a_again": (t * cdf).to(BF)}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What the passes give by the operators' definitions: the forward in 64 bits, and its gradients by differentiation."""
    s = prepare(case, seed)
    return _EXACT[case["path"]](s, case)


def _exact_attention(s, case):
    groups, w, S, tile, ahead = _attention_sizes(case)
    h, d = case["heads"], case["dim"]
    rel = [t.double().requires_grad_() for t in s["rel"]]
    sigma = s["sigma"].long().expand(groups, S)
    tile_of = torch.arange(S, device=DEV).div(tile, rounding_mode="floor")
    seen = (tile_of < ahead)[None, :] | (tile_of[None, :] == tile_of[:, None])
    dout = s["dout"].double().reshape(-1, h, d)
    dqkv = torch.empty(groups, S, 3, h, d, dtype=torch.float64, device=DEV)
    some = max(1, (1 << 26) // (h * S * S))
    heads = max(1, min(h, (1 << 27) // (S * S)))
    for g in range(0, groups, some):
        e = min(g + some, groups)
        row, col = sigma[g:e] // w, sigma[g:e] % w
        at_h, at_w = row[:, :, None] - row[:, None, :] + w - 1, col[:, :, None] - col[:, None, :] + w - 1
        for first in range(0, h, heads):
            part = slice(first, min(first + heads, h))
            qkv = s["qkv"][g:e, :, :, part].double().requires_grad_()
            q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))           # [g, heads, S, d]
            scores = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(d)
            for table, at in ((rel[0], at_h), (rel[1], at_w)):
                by_position = torch.matmul(q, table.t())
                scores = scores + by_position.gather(3, at[:, None].expand(-1, scores.shape[1], -1, -1))
            o = torch.matmul(torch.softmax(scores.masked_fill(~seen, -math.inf), 3), v).transpose(1, 2)
            if s["out_rows"] is None:
                upstream = dout.view(groups, S, h, d)[g:e, :, part]
            else:
                at = s["out_rows"][g:e].long()
                upstream = torch.where((at >= 0)[..., None, None], dout[at.clamp(min=0)], 0.0)[:, :, part]
            torch.autograd.backward(o, upstream)
            dqkv[g:e, :, :, part] = qkv.grad
    return {"dq": dqkv[:, :, 0], "dk": dqkv[:, :, 1], "dv": dqkv[:, :, 2], "drel_h": rel[0].grad, "drel_w": rel[1].grad}


def _exact_layernorm(s, case):
    idx = s["idx"].long().expand(case["batch"], -1)
    x, gamma = s["x"].double().requires_grad_(), s["gamma"].double().requires_grad_()
    beta = torch.zeros_like(gamma, requires_grad=True)
    rows = x.gather(1, idx.clamp(min=0)[..., None].expand(-1, -1, case["width"]))
    y = torch.nn.functional.layer_norm(rows, (case["width"],), gamma, beta, LN_EPS)
    y.backward(s["dy"].double() * (idx >= 0)[..., None])
    named = torch.zeros(x.shape[:2], dtype=torch.bool, device=DEV)
    b, p = torch.nonzero(idx >= 0, as_tuple=True)
    named[b, idx[b, p]] = True
    g0 = s["g0"].double()
    return {"dx": torch.where(named[..., None], g0 + x.grad, g0) if case["accumulate"] else torch.where(named[..., None], x.grad, g0),
            "dgamma": gamma.grad, "dbeta": beta.grad}


def _exact_values(x):
    """The values that x is held as: the nearest multiple, ties to even, of 1/127 of the largest magnitude in 64 columns."""
    out = torch.empty_like(x, dtype=torch.float64)
    for c in range(0, x.shape[1], COLS):
        part = x[:, c:c + COLS].double()
        step = part.abs().max(dim=1, keepdim=True)[0] / 127
        out[:, c:c + COLS] = torch.where(step > 0, torch.round(part / step) * step, 0.0)
    return out


def _exact_checkpoint(s, case):
    return {"x": _exact_values(s["x"])}


def _exact_gelu(s, case):
    gelu = torch.nn.functional.gelu
    t = _exact_values(s["x"]).requires_grad_()
    again = gelu(t)
    again.backward(s["da"].double())
    return {"a": gelu(s["x"].double()), "dh": t.grad, "a_again": again.detach()}


_PREPARE = {"attention": _prepare_attention, "layernorm": _prepare_layernorm, "checkpoint": _prepare_rows, "gelu": _prepare_rows}
_RUN = {"attention": _run_attention, "layernorm": _run_layernorm, "checkpoint": _run_checkpoint, "gelu": _run_gelu}
_EXACT = {"attention": _exact_attention, "layernorm": _exact_layernorm, "checkpoint": _exact_checkpoint, "gelu": _exact_gelu}
