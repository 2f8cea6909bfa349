"""Cases, plain forms and 64-bit values of the operators around the routing path of an MoE layer.

Four operators, each called as a program calls it:

route     router logits -> top-k expert ids and gate weights (softmax or sigmoid scores, a bias that only
          takes part in the choice, group-limited choice, renormalised weights), and the gradient of the
          logits from the gradient of the weights;
norm      residual addition and root-mean-square norm, to bf16 or to 8 bits (int8 or e4m3) with one scale per
          row, and the gradients of its input and of its weight;
quantize  bf16 rows to 8 bits with one scale per row (what the experts' second product reads);
matmul    the experts' products: 8-bit rows, grouped by expert as the routing layout orders them, times each
          expert's 8-bit weights, with a scale per row and per output channel; optionally gated
          (silu(gate) * up) in the same pass.

`own` selects the side: False computes the plain form in 32 bits with elementary torch operations, True calls
the framework.  Nothing of the framework is imported where `own` is false.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
CODE_MAX = {"int8": 127.0, "e4m3": 448.0}
CODE_TYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


# ---- cases --------------------------------------------------------------------------------------------------

def listed():
    return [
        # a handful of running requests: what one decoding step asks of the router (latency only)
        dict(name="route_step", op="route", grad=False, tokens=16, experts=256, topk=8, score="sigmoid", bias=True,
             n_group=8, topk_group=4, renorm=True, scale=2.5, logits="float32"),
        # the prefill batch of 16 ranks x 4096 tokens, biased sigmoid scores, 4 of 8 groups
        dict(name="route_prefill", op="route", grad=False, tokens=65536, experts=256, topk=8, score="sigmoid", bias=True,
             n_group=8, topk_group=4, renorm=True, scale=2.5, logits="float32"),
        # a training batch of 32 ranks x 512 tokens: softmax over 128 experts, gradient of bf16 logits
        dict(name="route_train", op="route", grad=True, tokens=16384, experts=128, topk=8, score="softmax", bias=False,
             n_group=1, topk_group=1, renorm=False, scale=1.0, logits="bfloat16"),
        # one decoding step of 128 requests: residual addition, norm, bf16 out
        dict(name="norm_step", op="norm", grad=False, rows=128, cols=7168, residual=True, out="bfloat16"),
        # the prefill batch, handed on in 8 bits
        dict(name="norm_prefill", op="norm", grad=False, rows=65536, cols=7168, residual=True, out="e4m3"),
        # backward pass of a training batch, the gradient of the residual stream added
        dict(name="norm_train", op="norm", grad=True, rows=16384, cols=4096, residual=True, out="bfloat16"),
        # the experts' inner rows of one decoding step (128 tokens, top-8), int8
        dict(name="quantize_step", op="quantize", rows=1024, cols=2048, out="int8"),
        # the same of a prefill chunk (16384 tokens, top-8), e4m3
        dict(name="quantize_prefill", op="quantize", rows=131072, cols=2048, out="e4m3"),
        # a single request on one rank's 32 experts: eight of them are read
        dict(name="matmul_one_token", op="matmul", tokens=1, experts=32, topk=8, inner=7168, channels=4096, gated=True,
             kind="int8", routing="uniform"),
        # a decoding step of 128 requests, gate and up projections: bound by the weights
        dict(name="matmul_step", op="matmul", tokens=128, experts=32, topk=8, inner=7168, channels=4096, gated=True,
             kind="int8", routing="uniform"),
        # a prefill chunk: bound by the products
        dict(name="matmul_prefill", op="matmul", tokens=2048, experts=32, topk=8, inner=7168, channels=4096, gated=True,
             kind="int8", routing="uniform"),
        # skewed routing, odd sizes, the second projection in e4m3
        dict(name="matmul_ragged", op="matmul", tokens=1237, experts=60, topk=6, inner=1424, channels=2040, gated=False,
             kind="e4m3", routing="zipf"),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["route", "norm", "quantize", "matmul", "matmul"])
    if op == "route":
        experts = rng.choice([8, 16, 60, 64, 96, 128, 160, 256, 384])
        sigmoid = rng.random() < 0.5
        groups = rng.choice([g for g in (1, 2, 4, 8) if experts % g == 0])
        keep = rng.randint((groups + 1) // 2, groups)
        topk = rng.randint(1, min(8, keep * (experts // groups)))
        return dict(op=op, grad=rng.random() < 0.4, tokens=min(_spread(rng, 1, 65536), 65536 * 256 // experts),
                    experts=experts, topk=topk, score="sigmoid" if sigmoid else "softmax", bias=sigmoid,
                    n_group=groups, topk_group=keep, renorm=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]),
                    logits=rng.choice(["float32", "bfloat16"]))
    if op == "norm":
        cols = rng.choice([1024, 4096, 7168, 8 * rng.randint(64, 1100)])
        return dict(op=op, grad=rng.random() < 0.4, rows=min(_spread(rng, 1, 65536), (1 << 28) // cols), cols=cols,
                    residual=rng.random() < 0.7, out=rng.choice(["bfloat16", "e4m3", "int8"]))
    if op == "quantize":
        cols = rng.choice([1024, 2048, 4096, 8 * rng.randint(32, 600)])
        return dict(op=op, rows=min(_spread(rng, 1, 131072), (1 << 28) // cols), cols=cols,
                    out=rng.choice(["e4m3", "e4m3", "int8"]))
    experts = rng.choice([8, 16, 24, 32, 60])
    inner = 16 * _spread(rng, 16, 448)
    channels = 2 * _spread(rng, 64, 2048)
    while experts * inner * channels > 32 * 7168 * 4096:
        channels = 2 * (channels // 4)
    topk = rng.randint(1, 8)
    return dict(op=op, tokens=_spread(rng, 1, 16384 // topk), experts=experts, topk=topk, inner=inner,
                channels=channels, gated=rng.random() < 0.5, kind=rng.choice(["int8", "e4m3"]),
                routing=rng.choice(["uniform", "zipf"]))


def work(case):
    if case["op"] == "route":
        n, e, k = case["tokens"], case["experts"], case["topk"]
        size = 4 if case["logits"] == "float32" else 2
        if case["grad"]:                                    # logits, ids and weight gradients in, logit gradients out
            return {"bytes": n * (2 * e * size + 8 * k), "flops": 6 * n * e}
        return {"bytes": n * (e * size + 8 * k) + (4 * e if case["bias"] else 0), "flops": 6 * n * e}
    if case["op"] == "norm":
        n, c, res = case["rows"], case["cols"], case["residual"]
        if case["grad"]:                                    # dy, h (and the residual's gradient) in, dx out; weight and its gradient
            return {"bytes": n * c * 2 * (4 if res else 3) + 6 * c, "flops": 12 * n * c}
        size = 2 if case["out"] == "bfloat16" else 1
        scale = 0 if case["out"] == "bfloat16" else 4
        return {"bytes": n * c * (2 * (3 if res else 1) + size) + n * scale + 2 * c, "flops": 6 * n * c}
    if case["op"] == "quantize":
        return {"bytes": case["rows"] * (case["cols"] * 3 + 4), "flops": 4 * case["rows"] * case["cols"]}
    e, k, t = case["experts"], case["topk"], case["tokens"]
    rows, inner, n = t * k, case["inner"], case["channels"]
    busy = e if case["routing"] == "uniform" and t * k > 8 * e else min(e, rows)
    if t == 1:
        busy = k
    wide = n // 2 if case["gated"] else n
    return {"bytes": rows * (inner + 4 + 2 * wide) + busy * n * (inner + 4), "flops": 2 * rows * inner * n}


# ---- inputs -------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


_contexts = {}


def _context(R, T, H, E, K):
    """A program makes one context for a shape and keeps it."""
    from paper_2607_26444_b200 import binding
    key = (R, T, H, E, K)
    if key not in _contexts:
        _contexts[key] = binding.MoEContext(R, T, H, E, K)
    return _contexts[key]


def _codes(values, kind):
    """Codes of values that are already in units of the scale."""
    if kind == "int8":
        return values.mul(32.0).round_().clamp_(-127, 127).to(torch.int8)
    return values.mul(64.0).clamp_(-448, 448).to(torch.float8_e4m3fn)


def _routing(case, g):
    """Distinct experts for every token: the k largest of E random keys, even or with Zipf popularity."""
    t, e, k = case["tokens"], case["experts"], case["topk"]
    keys = -torch.log(torch.rand((t, e), generator=g, device=DEV).clamp_(1e-9, 1 - 1e-7))
    if case["routing"] == "zipf":                           # exponential races: the smallest arrival times win
        order = torch.argsort(torch.rand(e, generator=g, device=DEV)).to(torch.float32)
        keys = keys * (order + 1.0) ** 1.2
    return torch.argsort(keys, dim=1)[:, :k].to(torch.int32).contiguous()


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"] == "route":
        n, e, k = case["tokens"], case["experts"], case["topk"]
        s["logits"] = _normal(g, n, e).to(getattr(torch, case["logits"]))
        s["bias"] = _normal(g, e).mul_(0.05) if case["bias"] else None
        if case["grad"]:                                    # the ids come from the forward pass, the gradient from combine
            s["ids"] = torch.argsort(torch.rand((n, e), generator=g, device=DEV), dim=1)[:, :k].to(torch.int32).contiguous()
            s["dw"] = _normal(g, n, k)
        if own:
            from paper_2607_26444_b200 import binding
            s["ctx"] = _context(1, n, 8, e, k)
            s["params"] = binding.make_route(case["score"], renormalise=case["renorm"], scale=case["scale"],
                                             n_group=case["n_group"], topk_group=case["topk_group"],
                                             group_score="top2" if case["score"] == "sigmoid" else "max")
            if case["grad"]:
                s["dlogits"] = torch.empty_like(s["logits"])
            else:
                s["ids"] = torch.empty((n, k), dtype=torch.int32, device=DEV)
                s["w"] = torch.empty((n, k), dtype=torch.float32, device=DEV)
    elif case["op"] == "norm":
        n, c = case["rows"], case["cols"]
        s["weight"] = (1.0 + 0.1 * _normal(g, c)).to(torch.bfloat16)
        s["x"] = _normal(g, n, c).to(torch.bfloat16)        # the layer's output; in the backward pass the stored sum
        if case["residual"]:
            s["residual"] = _normal(g, n, c).mul_(3.0).to(torch.bfloat16)
        if case["grad"]:
            s["dy"] = _normal(g, n, c).to(torch.bfloat16)
        if own:
            s["ctx"] = _context(1, 1, 8, 1, 1)
            s["y"] = torch.empty((n, c), dtype=torch.bfloat16, device=DEV)
            if case["grad"]:
                s["dweight"] = torch.empty(c, dtype=torch.float32, device=DEV)
                s["scratch"] = s["ctx"].norm_grad_scratch(n, c)
            elif case["residual"]:
                s["h"] = torch.empty((n, c), dtype=torch.bfloat16, device=DEV)
            if case["out"] in CODE_TYPE:
                s["q"] = torch.empty((n, c), dtype=CODE_TYPE[case["out"]], device=DEV)
                s["scale"] = torch.empty(n, dtype=torch.float32, device=DEV)
    elif case["op"] == "quantize":
        n, c = case["rows"], case["cols"]
        s["x"] = _normal(g, n, c).mul_(0.5 + torch.rand((n, 1), generator=g, device=DEV)).to(torch.bfloat16)
        if own:
            s["ctx"] = _context(1, 1, 8, 1, 1)
            s["y"] = torch.empty((n, c), dtype=torch.bfloat16, device=DEV)
            s["q"] = torch.empty((n, c), dtype=CODE_TYPE[case["out"]], device=DEV)
            s["scale"] = torch.empty(n, dtype=torch.float32, device=DEV)
    else:
        e, inner, n = case["experts"], case["inner"], case["channels"]
        rows = case["tokens"] * case["topk"]
        ids = _routing(case, g)
        s["count"] = torch.bincount(ids.reshape(-1).long(), minlength=e)
        s["most"] = int(s["count"].max())                   # rows of the busiest expert
        s["a"] = _codes(_normal(g, rows, inner), case["kind"])
        s["w"] = torch.empty((e, n, inner), dtype=CODE_TYPE[case["kind"]], device=DEV)
        for i in range(e):
            s["w"][i] = _codes(_normal(g, n, inner), case["kind"])
        unit = 32.0 if case["kind"] == "int8" else 64.0
        s["a_scale"] = (0.5 + torch.rand(rows, generator=g, device=DEV)) / unit
        s["w_scale"] = (0.5 + torch.rand((e, n), generator=g, device=DEV)) / (unit * math.sqrt(inner))
        if own:
            s["ctx"] = _context(1, case["tokens"], 8, e, case["topk"])
            s["layout"] = s["ctx"].layout(ids)
            s["out"] = torch.empty((rows, n // 2 if case["gated"] else n), dtype=torch.bfloat16, device=DEV)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    if case["op"] == "route":
        if case["grad"]:
            ctx.route_grad(s["params"], s["logits"], s["ids"], s["dw"], s["dlogits"])
            return {"dlogits": s["dlogits"]}
        ctx.route(s["params"], s["logits"], s["ids"], s["w"], bias=s["bias"])
        return {"ids": s["ids"], "w": s["w"]}
    if case["op"] == "norm" and case["grad"]:
        ctx.norm_grad(s["dy"], s["x"], s["weight"], EPS, s["y"], s["dweight"], dresidual=s.get("residual"),
                      scratch=s["scratch"])
        return {"dx": s["y"], "dweight": s["dweight"]}
    if case["op"] == "norm":
        q = case["out"] in CODE_TYPE
        ctx.norm(s["x"], s["weight"], EPS, out=None if q else s["y"], residual=s.get("residual"),
                 residual_out=s.get("h"), q=s.get("q"), q_scale=s.get("scale"))
        got = _quantized(s) if q else {"y": s["y"]}
        return {**got, "h": s["h"]} if case["residual"] else got
    if case["op"] == "quantize":
        ctx.quantize_rows(s["x"], s["q"], s["scale"])
        return _quantized(s)
    ctx.expert_matmul(s["layout"], s["a"], s["a_scale"], s["w"], s["w_scale"], s["out"], gated=case["gated"])
    return {"y": s["out"]}


def _quantized(s):
    """e4m3 codes are values by themselves; int8 codes are given as the values they stand for."""
    if s["q"].dtype == torch.int8:
        torch.mul(s["q"], s["scale"][:, None], out=s["y"])
        return {"y": s["y"], "scale": s["scale"]}
    return {"q": s["q"], "scale": s["scale"]}


def _run_plain(s):
    case = s["case"]
    if case["op"] == "route":
        return _plain_route_grad(s) if case["grad"] else _plain_route(s)
    if case["op"] == "norm":
        return _plain_norm_grad(s) if case["grad"] else _plain_norm(s)
    if case["op"] == "quantize":
        return _plain_codes(s["x"].float(), case["out"])
    return _plain_matmul(s)


def _plain_scores(logits, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-logits))
    p = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    return p / p.sum(dim=1, keepdim=True)


def _plain_route(s):
    case = s["case"]
    n, e, k, groups = case["tokens"], case["experts"], case["topk"], case["n_group"]
    logits = s["logits"].float()
    scores = _plain_scores(logits, case["score"])
    choice = logits if s["bias"] is None else scores + s["bias"]     # without a bias scores order as logits do
    if groups > 1:
        inside = torch.sort(choice.view(n, groups, e // groups), dim=2, descending=True).values
        two = case["score"] == "sigmoid" and e // groups > 1
        best = inside[:, :, 0] + inside[:, :, 1] if two else inside[:, :, 0]
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :case["topk_group"]]
        out = torch.ones((n, groups), dtype=torch.bool, device=DEV).scatter_(1, kept, False)
        choice = choice.masked_fill(out.repeat_interleave(e // groups, dim=1), -math.inf)
    ids = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :k]
    w = scores.gather(1, ids)
    if case["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    return {"ids": ids.to(torch.int32), "w": w * case["scale"]}


def _plain_route_grad(s):
    case = s["case"]
    scores = _plain_scores(s["logits"].float(), case["score"])
    ids = s["ids"].long()
    chosen, ds = scores.gather(1, ids), s["dw"] * case["scale"]
    if case["renorm"]:
        total = chosen.sum(dim=1, keepdim=True)
        ds = (ds - (ds * chosen).sum(dim=1, keepdim=True) / total) / total
    full = torch.zeros_like(scores).scatter_(1, ids, ds)
    if case["score"] == "sigmoid":
        d = full * scores * (1.0 - scores)
    else:
        d = scores * (full - (full * scores).sum(dim=1, keepdim=True))
    return {"dlogits": d.to(s["logits"].dtype)}


def _plain_norm(s):
    case = s["case"]
    h = s["x"].float()
    if case["residual"]:                                    # the sum is stored in bf16, and what is stored is normed
        stored = (h + s["residual"].float()).to(torch.bfloat16)
        h = stored.float()
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * s["weight"].float()
    got = {"y": y.to(torch.bfloat16)} if case["out"] == "bfloat16" else _plain_codes(y, case["out"])
    return {**got, "h": stored} if case["residual"] else got


def _plain_codes(y, kind):
    scale = y.abs().amax(dim=1, keepdim=True) / CODE_MAX[kind]
    q = y / torch.where(scale == 0, torch.ones_like(scale), scale)
    if kind == "int8":
        return {"y": (torch.round(q) * scale).to(torch.bfloat16), "scale": scale[:, 0]}
    return {"q": q.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn), "scale": scale[:, 0]}


def _plain_norm_grad(s):
    h, dy, w = s["x"].float(), s["dy"].float(), s["weight"].float()
    rstd = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
    hat, g = h * rstd, dy * w
    dx = rstd * (g - hat * (g * hat).mean(dim=1, keepdim=True))
    if s["case"]["residual"]:
        dx = dx + s["residual"].float()
    return {"dx": dx.to(torch.bfloat16), "dweight": (dy * hat).sum(dim=0)}


def _grouped(s):
    """(expert, place inside its segment) of every row: rows are ordered by expert."""
    end = torch.cumsum(s["count"], 0)
    rows = s["a"].shape[0]
    row = torch.arange(rows, device=DEV)
    expert = torch.searchsorted(end, row, right=True)
    return expert, row - (end - s["count"])[expert]


def _products(s, dtype):
    """Rows times their expert's weights, both unscaled, through one padded batch of products."""
    case = s["case"]
    expert, place = _grouped(s)
    padded = torch.zeros((case["experts"], s["most"], case["inner"]), dtype=dtype, device=DEV)
    padded[expert, place] = s["a"].to(dtype)
    return torch.bmm(padded, s["w"].to(dtype).transpose(1, 2))[expert, place], expert


def _plain_matmul(s):
    case = s["case"]
    acc, expert = _products(s, torch.float32)
    y = acc * s["a_scale"][:, None] * s["w_scale"][expert]
    if case["gated"]:
        gate, up = y[:, :case["channels"] // 2], y[:, case["channels"] // 2:]
        y = gate / (1.0 + torch.exp(-gate)) * up
    return {"y": y.to(torch.bfloat16)}


# ---- the definition in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    with_own = globals()["own"]
    globals()["own"] = False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = with_own
    return {"route": _exact_route, "norm": _exact_norm, "quantize": _exact_quantize, "matmul": _exact_matmul}[case["op"]](s)


def _exact_weights(case, scores, ids):
    w = torch.take_along_dim(scores, ids, dim=1)
    return case["scale"] * (w / w.sum(1, keepdim=True) if case["renorm"] else w)


def _exact_route(s):
    case = s["case"]
    logits = s["logits"].double().requires_grad_(case["grad"])
    scores = torch.sigmoid(logits) if case["score"] == "sigmoid" else torch.softmax(logits, 1)
    if case["grad"]:
        w = _exact_weights(case, scores, s["ids"].long())
        (w * s["dw"].double()).sum().backward()
        return {"dlogits": logits.grad}
    choice = scores if s["bias"] is None else scores + s["bias"].double()
    n, g = case["tokens"], case["n_group"]
    inside = choice.view(n, g, -1)
    two = min(inside.shape[2], 2 if case["score"] == "sigmoid" else 1)
    best = inside.topk(two, dim=2).values.sum(2)
    least = best.topk(case["topk_group"], dim=1).values[:, -1:]
    choice = torch.where((best >= least)[:, :, None].expand_as(inside).reshape(n, -1), choice, -math.inf)
    if case["logits"] == "bfloat16" and s["bias"] is None:
        return None                                         # equal logits: the order of ties is not a value
    return {"ids": None, "w": _exact_weights(case, scores, choice.topk(case["topk"], dim=1).indices)}


def _exact_row_codes(y, kind):
    top = y.abs().max(1).values
    scale = top / CODE_MAX[kind]
    units = y / torch.where(top == 0, 1.0, scale)[:, None]
    if kind == "int8":
        return {"y": units.round() * scale[:, None], "scale": scale}
    return {"q": units.float().to(torch.float8_e4m3fn).double(), "scale": scale}


def _exact_norm(s):
    case = s["case"]
    w = s["weight"].double()
    if case["grad"]:
        h = s["x"].double().requires_grad_()
        w = w.requires_grad_()
        y = w * h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS)
        y.backward(s["dy"].double())
        dx = h.grad + s["residual"].double() if case["residual"] else h.grad
        return {"dx": dx, "dweight": w.grad}
    h = s["x"].double()
    if case["residual"]:
        full = h + s["residual"].double()
        h = full.to(torch.bfloat16).double()
    y = w * h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS)
    got = {"y": y} if case["out"] == "bfloat16" else _exact_row_codes(y, case["out"])
    return {**got, "h": full} if case["residual"] else got


def _exact_quantize(s):
    return _exact_row_codes(s["x"].double(), s["case"]["out"])


def _exact_matmul(s):
    acc, expert = _products(s, torch.float64)
    y = acc * (s["a_scale"].double()[:, None] * s["w_scale"].double()[expert])
    if s["case"]["gated"]:
        gate, up = y.chunk(2, dim=1)
        y = torch.nn.functional.silu(gate) * up
    return {"y": y}
