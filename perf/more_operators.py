"""Contractions in 8 bits and the step between two halves of a block, as calls of the library and in plain form: how fast each is, and how far off.

A case is a dict of plain values.  Its ``path`` says which operators it stands for:

  product     a Linear layer in 8-bit integers: bf16 tokens to codes with a scale for each (``ssam_quantize_rows``), and their product with
              a weight that is held as codes with a scale for each output channel (``ssam_linear_i8``).  ``epilogue``: ``bias``, ``gelu``,
              ``scatter`` or ``add``; the last two write, or add to, rows of a map, ``tokens`` of them an image (a map longer than that
              has slots without a token, as the padded windows of a grid do)
  residual    what lies between two halves of a block: the branch behind its own LayerNorm (``post``), times a gate (of the features, or of
              every image's features), joins the scaled residual stream, whose LayerNorm goes to the rows that the next half reads
              (``ssam_residual_norm``).  ``branch`` and ``out``: the order of the branch's rows and of the result's: ``windows`` of
              14 x 14 with padding slots, the ``kept`` tokens of every image, or ``all`` in their own order (``out`` also ``none``).
              With ``features`` the result is written in 8 bits (``ssam_residual_norm_i8``) and multiplied (``ssam_linear_i8``)
  gradient    the gradients of ``residual`` (``ssam_residual_norm_backward``): of the stream, the branch, the gate and both LayerNorms
"""
import math

import torch

own = False

DEV = "cuda"
BF = torch.bfloat16
STRIPE, WINDOW = 4, 14     # G of the stripe interleave; side of a window
LN_EPS = 1e-6
ALPHA = 0.9375             # what the residual stream is scaled by


def listed():
    return [
        # qkv of one token, as a prompt's or a classifier's: the least that a program asks for, bound by latency and by the weight's bytes
        dict(name="product_one_token", path="product", batch=1, rows=1, K=1280, N=3840, epilogue="bias", tokens=0),
        # fc1 of the kept tokens of a small image, large width
        dict(name="product_kept_fc1", path="product", batch=1, rows=313, K=1024, N=4096, epilogue="gelu", tokens=0),
        # a stage of a hierarchical encoder: no multiple of a tile anywhere
        dict(name="product_stage_144", path="product", batch=1, rows=4900, K=144, N=576, epilogue="bias", tokens=0),
        # the output projection of one image's windows, back to the tokens' own order: 804 slots of 4900 are padding
        dict(name="product_proj_b1", path="product", batch=1, rows=4900, K=1280, N=1280, epilogue="add", tokens=4096),
        # fc2 of the kept tokens of a batch, added into the residual stream
        dict(name="product_fc2_b8", path="product", batch=8, rows=1638, K=5120, N=1280, epilogue="add", tokens=4096),
        # qkv of a batch at the huge width: the largest
        dict(name="product_qkv_b8", path="product", batch=1, rows=32768, K=1280, N=3840, epilogue="bias", tokens=0),
        # one small image, dense: both halves in the tokens' own order
        dict(name="residual_28x28", path="residual", batch=1, grid=28, width=768, branch="all", out="all", post=True, gate="features", density=1.0, features=0),
        # a batch behind its windows' attention: the kept tokens go on to the MLP
        dict(name="residual_windows_b8", path="residual", batch=8, grid=64, width=1280, branch="windows", out="kept", post=True, gate="features", density=0.4, features=0),
        # a batch behind its MLP, gates of every image: the next block's windows, in 8 bits, and their qkv
        dict(name="residual_to_qkv_b4", path="residual", batch=4, grid=64, width=1024, branch="kept", out="windows", post=False, gate="images", density=0.4, features=1536),
        # training: a small image, and a branch without a LayerNorm of its own on a grid that windows do not divide
        dict(name="gradient_28x28", path="gradient", batch=1, grid=28, width=768, branch="all", out="all", post=True, gate="features", density=1.0),
        dict(name="gradient_50x50_b2", path="gradient", batch=2, grid=50, width=1152, branch="kept", out="windows", post=False, gate="images", density=0.5),
        # training: a batch at the huge width
        dict(name="gradient_windows_b8", path="gradient", batch=8, grid=64, width=1280, branch="windows", out="kept", post=True, gate="features", density=0.4),
    ]


def draw(rng):
    """One more case of the same ranges: products of one to 32768 tokens, 16 to 5120 features in and 8 to 5120 out; steps on grids of one token to
    64 x 64, 16 to 2048 features wide, with every order, gate and norm."""
    between = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        path = rng.choice(["product", "product", "residual", "gradient"])
        if path == "product":
            epilogue = rng.choice(["bias", "gelu", "scatter", "add"])
            mapped = epilogue in ("scatter", "add")
            batch = between(1, 8) if mapped else 1
            rows = between(1, 32768 // batch)
            case = dict(path=path, batch=batch, rows=rows, K=rng.choice([768, 1024, 1280, 16 * between(1, 320)]), N=rng.choice([1280, 2304, 8 * between(1, 640)]),
                        epilogue=epilogue, tokens=max(1, min(4096, int(rows * rng.choice([0.8, 1.0, 2.5])))) if mapped else 0)
        else:
            case = dict(path=path, batch=between(1, 8), grid=between(1, 64), width=rng.choice([768, 1024, 1280, 16 * between(1, 128)]),
                        branch=rng.choice(["windows", "kept", "all"]), out=rng.choice(["windows", "kept", "all", "none"]), post=rng.random() < 0.6,
                        gate=rng.choice(["none", "features", "images"]), density=rng.choice([0.1, 0.3, 0.4, 0.7, 1.0]))
            if path == "residual":
                case["features"] = rng.choice([0, 0, 8 * between(1, 192)]) if case["out"] != "none" else 0
        if _cost(case) <= _MOST[path]:
            return case


# ------------------------------------------------------------------ sizes
def _kept(case):
    n = case["grid"] ** 2
    return max(1, min(n, int(math.floor(case["density"] * n + 1e-6))))


def _rows_of(case, which):
    """-> rows of an image, and how many of them have a token"""
    n = case["grid"] ** 2
    if which == "none":
        return 0, 0
    if which == "kept":
        return _kept(case), _kept(case)
    return (n, n) if which == "all" else (_side(case["grid"]) ** 2 * _window(case["grid"]) ** 2, n)


def _window(grid):
    return min(WINDOW, grid)


def _side(grid):
    return -(-grid // _window(grid))


def work(case):
    """Bytes (inputs and outputs once) and flops of one pass."""
    if case["path"] == "product":
        M, N, K = case["batch"] * case["rows"], case["N"], case["K"]
        stored = M if not case["tokens"] else case["batch"] * min(case["rows"], case["tokens"])
        return {"bytes": 2.0 * M * K + N * K + 8.0 * N + 2.0 * stored * N * (2 if case["epilogue"] == "add" else 1) + (4.0 * M if case["tokens"] else 0), "flops": 2.0 * M * N * K}
    B, n, D = case["batch"], case["grid"] ** 2, case["width"]
    branch, out = B * _rows_of(case, case["branch"])[1], B * _rows_of(case, case["out"])[1]
    rows, qkv = B * _rows_of(case, case["out"])[0], case.get("features", 0)
    if case["path"] == "residual":
        got = 2.0 * out * D if not qkv else 1.0 * qkv * D + 2.0 * rows * qkv
        return {"bytes": 2.0 * D * (2 * B * n + branch) + got, "flops": 30.0 * B * n * D + 2.0 * rows * D * qkv}
    return {"bytes": 2.0 * D * (3 * B * n + 2 * branch + out) + 20.0 * D, "flops": 60.0 * B * n * D}


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 100


#: no drawn case is more work than the largest listed one of its path
_MOST = {}
for _c in listed():
    _MOST[_c["path"]] = max(_MOST.get(_c["path"], 0.0), _cost(_c))


# ------------------------------------------------------------------ inputs
def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(dtype)


def _some(gen, batch, n, k):
    """[batch, k]: k of n tokens of every image, in their order"""
    return torch.rand(batch, n, generator=gen, device=DEV).argsort(dim=1)[:, :k].sort(dim=1)[0]


def _token_rows(gen, case, which):
    """[batch or 1, rows]: the token of every row, -1 where it has none"""
    g = case["grid"]
    if which == "kept":
        return _some(gen, case["batch"], g * g, _kept(case))
    if which == "all":
        return torch.arange(g * g, device=DEV)[None]
    w, side = _window(g), _side(g)
    at = torch.arange(side, device=DEV)[:, None] * w + torch.arange(w, device=DEV)            # [side, w]
    row, col = at[:, None, :, None], at[None, :, None, :]
    token = torch.where((row < g) & (col < g), row * g + col, -1).reshape(side * side, w * w)
    if w * w % STRIPE == 0:
        token = token.view(-1, w * w // STRIPE, STRIPE).transpose(1, 2)
    return token.reshape(1, -1)


def _row_of_token(rows, n):
    """The inverse: [batch or 1, n], the row of every token, -1 where it has none"""
    out = torch.full((rows.shape[0], n + 1), -1, device=DEV)
    at = torch.arange(rows.shape[1], device=DEV).expand_as(rows)
    return out.scatter_(1, torch.where(rows >= 0, rows, n), at)[:, :n].to(torch.int32).contiguous()


def _weight_codes(gen, N, K):
    """What a program holds a weight as from its loading on: codes, and a scale for each output channel."""
    w = _normal(gen, N, K, std=0.02) * torch.exp(_normal(gen, N, 1, std=0.3))
    top = w.abs().amax(1, keepdim=True)
    return torch.round(w * (127 / top)).to(torch.int8), (top / 127)[:, 0].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return {"case": case, **_PREPARE[case["path"]](case, gen)}


def _prepare_product(case, gen):
    batch, rows, K, N = case["batch"], case["rows"], case["K"], case["N"]
    # activations: every feature has a size of its own, as trained networks have, and every token too
    x = _normal(gen, batch * rows, K) * torch.exp(_normal(gen, K, std=0.5)) * torch.exp(_normal(gen, batch * rows, 1, std=0.3))
    w, w_scales = _weight_codes(gen, N, K)
    s = {"x": x.to(BF), "w": w, "w_scales": w_scales, "bias": _normal(gen, N, std=0.5), "map": None, "out": None}
    if case["tokens"]:
        n = case["tokens"]
        where = torch.full((batch, rows), -1, device=DEV)
        slots = _some(gen, batch, rows, min(rows, n))
        where.scatter_(1, slots, torch.rand(batch, n, generator=gen, device=DEV).argsort(dim=1)[:, :min(rows, n)])
        s["map"] = where.to(torch.int32)
        s["out"] = _normal(gen, batch * n, N, dtype=BF)
    return s


def _prepare_step(case, gen):
    batch, n, D = case["batch"], case["grid"] ** 2, case["width"]
    branch = _token_rows(gen, case, case["branch"])
    s = {"x": _normal(gen, batch, n, D, dtype=BF) + _normal(gen, 1, 1, D, std=0.5, dtype=BF),
         "o": _normal(gen, batch, branch.shape[1], D, std=0.7, dtype=BF), "src": _row_of_token(branch, n),
         "post": (1 + _normal(gen, D, std=0.1), _normal(gen, D, std=0.1)) if case["post"] else None,
         "gate": None if case["gate"] == "none" else 0.3 + _normal(gen, *((batch, D) if case["gate"] == "images" else (D,)), std=0.1),
         "pre": None, "dst": None, "rows": 0}
    if case["out"] != "none":
        out = _token_rows(gen, case, case["out"])
        s |= {"pre": (1 + _normal(gen, D, std=0.1), _normal(gen, D, std=0.1)), "dst": _row_of_token(out, n), "rows": out.shape[1]}
    return s


def _prepare_residual(case, gen):
    s, D = _prepare_step(case, gen), case["width"]
    if case["features"]:
        # rows without a token are zeros from the start, and stay so
        w, w_scales = _weight_codes(gen, case["features"], D)
        s |= {"codes": torch.zeros(case["batch"], s["rows"], D, dtype=torch.int8, device=DEV), "scales": torch.zeros(case["batch"], s["rows"], device=DEV),
              "w": w, "w_scales": w_scales, "bias": _normal(gen, case["features"], std=0.5)}
    elif s["pre"]:
        s["y"] = torch.zeros(case["batch"], s["rows"], D, dtype=BF, device=DEV)
    return s


def _prepare_gradient(case, gen):
    s, D = _prepare_step(case, gen), case["width"]
    s["dx"] = _normal(gen, *s["x"].shape, std=0.02, dtype=BF)
    s["dy"] = _normal(gen, case["batch"], s["rows"], D, std=0.02, dtype=BF) if s["pre"] else None
    s["do"] = torch.zeros_like(s["o"])                             # rows without a token have no gradient
    return s


# ------------------------------------------------------------------ passes
def run(state):
    return _RUN[state["case"]["path"]](state, state["case"])


def _codes(x):
    """fp32 rows -> whole numbers of -127 to 127, and the scale of every row.  In 64 bits: half of a row's largest value is a tie."""
    top = x.abs().amax(1, keepdim=True).double()
    codes = torch.round(x.double() * torch.where(top > 0, 127 / top, 0.0))
    return codes.float(), (top / 127).clamp(min=2.0 ** -126).float()


def _linear(codes, scales, s):
    return (codes @ s["w"].float().t()) * s["w_scales"] * scales + s["bias"]


def _run_product(s, case):
    if own:
        from paper_2605_17633_amd import binding as B
        codes, scales = B.ssam_quantize_rows(s["x"])
        epilogue = {"bias": B.EPI_BIAS, "gelu": B.EPI_BIAS_GELU, "scatter": B.EPI_BIAS_SCATTER, "add": B.EPI_BIAS_SCATTER_ADD}[case["epilogue"]]
        if not case["tokens"]:
            return {"y": B.ssam_linear_i8(codes, scales, s["w"], s["w_scales"], s["bias"], epilogue=epilogue)}
        return {"y": B.ssam_linear_i8(codes, scales, s["w"], s["w_scales"], s["bias"], s["out"], epilogue=epilogue, row_map=s["map"], rows_per_batch=case["rows"],
                                      map_batch_stride=case["rows"], dst_rows_per_batch=case["tokens"])}
    y = _linear(*_codes(s["x"].float()), s)
    if case["epilogue"] == "gelu":
        y = 0.5 * y * torch.erfc(y * -math.sqrt(0.5))
    if not case["tokens"]:
        return {"y": y.to(BF)}
    image, slot = torch.nonzero(s["map"] >= 0, as_tuple=True)
    to, y = image * case["tokens"] + s["map"][image, slot].long(), y[image * case["rows"] + slot]
    s["out"][to] = (y + s["out"][to].float() if case["epilogue"] == "add" else y).to(BF)
    return {"y": s["out"]}


def _normalised(v):
    """Rows less their mean over their deviation, and one over that"""
    v = v - v.mean(1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + LN_EPS)
    return v * rstd, rstd


def _pairs(which, batch, rows):
    """[batch or 1, n] rows of tokens -> the tokens (of all images) that have one, their images, and those rows (of all images)"""
    image, token = torch.nonzero(which.expand(batch, -1) >= 0, as_tuple=True)
    return image * which.shape[1] + token, image, image * rows + which.expand(batch, -1)[image, token].long()


def _gate(s, image):
    g = s["gate"]
    return 1.0 if g is None else g[image] if g.dim() == 2 else g


def _run_residual(s, case):
    qkv = case["features"]
    if own:
        from paper_2605_17633_amd import binding as B
        step = dict(o=s["o"], src=s["src"], post=s["post"], gate=s["gate"], alpha=ALPHA, pre=s["pre"], dst=s["dst"], eps=LN_EPS)
        if not qkv:
            x, y = B.ssam_residual_norm(s["x"], **step, y=s.get("y"))
            return {"x": x, "y": y}
        x, codes, scales = B.ssam_residual_norm_i8(s["x"], **step, codes=s["codes"], scales=s["scales"])
        return {"x": x, "y": B.ssam_linear_i8(codes.view(-1, case["width"]), scales.view(-1), s["w"], s["w_scales"], s["bias"])}
    batch, n, D = s["x"].shape
    token, image, row = _pairs(s["src"], batch, s["o"].shape[1])
    branch = s["o"].view(-1, D)[row].float()
    if s["post"]:
        branch = _normalised(branch)[0] * s["post"][0] + s["post"][1]
    x = s["x"].view(-1, D).clone()
    x[token] = (ALPHA * x[token].float() + _gate(s, image) * branch).to(BF)
    if not s["pre"]:
        return {"x": x.view(batch, n, D), "y": None}
    token, image, row = _pairs(s["dst"], batch, s["rows"])
    y = _normalised(x[token].float())[0] * s["pre"][0] + s["pre"][1]
    if not qkv:
        s["y"].view(-1, D)[row] = y.to(BF)
        return {"x": x.view(batch, n, D), "y": s["y"]}
    codes, scales = _codes(y)
    s["codes"].view(-1, D)[row] = codes.to(torch.int8)
    s["scales"].view(-1)[row] = scales[:, 0]
    return {"x": x.view(batch, n, D), "y": _linear(s["codes"].view(-1, D).float(), s["scales"].view(-1, 1), s).to(BF)}


def _run_gradient(s, case):
    if own:
        from paper_2605_17633_amd import binding as B
        dx, do, dgate, dpost, dpre = B.ssam_residual_norm_backward(s["x"], o=s["o"], src=s["src"], post=s["post"], gate=s["gate"], alpha=ALPHA, pre=s["pre"], dst=s["dst"],
                                                                   eps=LN_EPS, dy=s["dy"], dx_out=s["dx"], do=s["do"])
        return {"dx": dx, "do": do, "dgate": dgate, "dpost": dpost, "dpre": dpre}
    batch, n, D = s["x"].shape
    back = lambda g, h, rstd: (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * rstd  # noqa: E731
    total = lambda t: t.sum(0, dtype=torch.float64).float()  # noqa: E731
    grad, dpre, dgate, dpost = s["dx"].view(-1, D).float(), None, None, None
    if s["pre"]:
        token, image, row = _pairs(s["dst"], batch, s["rows"])
        h, rstd = _normalised(s["x"].view(-1, D)[token].float())
        dy = s["dy"].view(-1, D)[row].float()
        dpre = (total(dy * h), total(dy))
        grad[token] += back(dy * s["pre"][0], h, rstd)
    token, image, row = _pairs(s["src"], batch, s["o"].shape[1])
    g, o = grad[token], s["o"].view(-1, D)[row].float()
    grad[token] *= ALPHA
    do = g * _gate(s, image)
    h, rstd = _normalised(o) if s["post"] else (o, None)
    if s["gate"] is not None:
        times = g * (h * s["post"][0] + s["post"][1] if s["post"] else o)
        if s["gate"].dim() == 1:
            dgate = total(times)
        else:
            dgate = torch.zeros(batch * n, D, device=DEV).index_copy_(0, token, times).view(batch, n, D).sum(1, dtype=torch.float64).float()
    if s["post"]:
        dpost = (total(do * h), total(do))
        do = back(do * s["post"][0], h, rstd)
    s["do"].view(-1, D)[row] = do.to(BF)
    return {"dx": grad.view(batch, n, D).to(BF), "do": s["do"], "dgate": dgate, "dpost": dpost, "dpre": dpre}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What the passes give by the operators' definitions: the forward in 64 bits, and its gradients by differentiation."""
    s = prepare(case, seed)
    return _EXACT[case["path"]](s, case)


def _exact_values(x):
    """The values that rows are held as: the nearest multiple, ties to even, of 1/127 of a row's largest magnitude."""
    top = x.double().abs().max(dim=1, keepdim=True)[0]
    return torch.where(top > 0, torch.round(x.double() / top * 127) * top / 127, 0.0)


def _exact_linear(values, s):
    return torch.nn.functional.linear(values, s["w"].double() * s["w_scales"].double()[:, None], s["bias"].double())


def _exact_product(s, case):
    y = _exact_linear(_exact_values(s["x"]), s)
    if case["epilogue"] == "gelu":
        y = torch.nn.functional.gelu(y)
    if not case["tokens"]:
        return {"y": y}
    out = s["out"].double().view(case["batch"], -1, case["N"])
    y = y.view(case["batch"], case["rows"], -1)
    for b in range(case["batch"]):
        there = s["map"][b] >= 0
        to = s["map"][b][there].long()
        out[b, to] = y[b, there] + out[b, to] if case["epilogue"] == "add" else y[b, there]
    return {"y": out.view(-1, case["N"])}


def _step_by_definition(s, case, x, o, gate, post, pre):
    """One image after the other; x as the forward call is given it -> the new stream and LN of it for every token"""
    D, new, ys = case["width"], [], []
    for b in range(case["batch"]):
        src = s["src"][b % s["src"].shape[0]].long()
        n = o[b][src.clamp(min=0)]
        if post:
            n = torch.nn.functional.layer_norm(n, (D,), *post, LN_EPS)
        if gate is not None:
            n = n * (gate[b] if gate.dim() == 2 else gate)
        new.append(torch.where((src >= 0)[:, None], ALPHA * x[b] + n, x[b]))
    return torch.stack(new)


def _exact_residual(s, case):
    doubles = lambda t: None if t is None else tuple(v.double() for v in t) if isinstance(t, tuple) else t.double()  # noqa: E731
    x = _step_by_definition(s, case, *(doubles(s[k]) for k in ("x", "o", "gate", "post", "pre")))
    if not s["pre"]:
        return {"x": x, "y": None}
    # the LayerNorm is that of the stream as it is stored
    y = torch.nn.functional.layer_norm(x.to(BF).double(), x.shape[2:], *doubles(s["pre"]), LN_EPS)
    out = torch.zeros(case["batch"], s["rows"], case["width"], dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        dst = s["dst"][b % s["dst"].shape[0]].long()
        out[b, dst[dst >= 0]] = y[b][dst >= 0]
    if not case["features"]:
        return {"x": x, "y": out}
    return {"x": x, "y": _exact_linear(_exact_values(out.flatten(0, 1)), s)}


def _exact_gradient(s, case):
    leaf = lambda t: None if t is None else tuple(leaf(v) for v in t) if isinstance(t, tuple) else t.double().requires_grad_()  # noqa: E731
    grad = lambda t: None if t is None else tuple(v.grad for v in t) if isinstance(t, tuple) else t.grad  # noqa: E731
    o, gate, post, pre = (leaf(s[k]) for k in ("o", "gate", "post", "pre"))
    # the stream behind the step is given; what it was in front of it does not matter to any gradient
    before = torch.zeros_like(s["x"], dtype=torch.float64, requires_grad=True)
    after = _step_by_definition(s, case, before, o, gate, post, pre)
    upstream = s["dx"].double()
    if pre:
        x = s["x"].double().requires_grad_()
        y = torch.nn.functional.layer_norm(x, x.shape[2:], *pre, LN_EPS)
        dy = torch.zeros_like(y)
        for b in range(case["batch"]):
            dst = s["dst"][b % s["dst"].shape[0]].long()
            dy[b, dst >= 0] = s["dy"][b, dst[dst >= 0]].double()
        y.backward(dy)
        upstream = upstream + x.grad
    after.backward(upstream)
    return {"dx": before.grad, "do": o.grad, "dgate": grad(gate), "dpost": grad(post), "dpre": grad(pre)}


_PREPARE = {"product": _prepare_product, "residual": _prepare_residual, "gradient": _prepare_gradient}
_RUN = {"product": _run_product, "residual": _run_residual, "gradient": _run_gradient}
_EXACT = {"product": _exact_product, "residual": _exact_residual, "gradient": _exact_gradient}
