"""Cases, plain forms and 64-bit values of the experts' 4-bit path and of the router's balance loss.

Three operators, each called as a program calls it:

rows4     bf16 rows to 4-bit codes (e2m1) with a scale per block of a row, and back to the values that the codes
          stand for: mxfp4 (blocks of 32, a power of two each) or nvfp4 (blocks of 16, an e4m3 scale each, and
          one fp32 scale per row);
matmul4   the experts' products: 4-bit rows, grouped by expert as the routing layout orders them, times each
          expert's 4-bit weights, both with their block scales; optionally gated (silu(gate) * up) in the pass;
balance   the balance loss of a router's batch and the mean square of its log-sum-exp, the counts per expert, and
          the gradient of the logits: one training step of the router, over the batch or per source rank.

`own` selects the side: False computes the plain form in 32 bits with elementary torch operations, True calls
the framework.  Nothing of the framework is imported where `own` is false.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = {"mxfp4": 32, "nvfp4": 16}                  # values that share a scale
SCALE_TYPE = {"mxfp4": torch.float8_e8m0fnu, "nvfp4": torch.float8_e4m3fn}
CODE_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]          # of codes 0..7; bit 3 is the sign
MIDPOINTS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
WEIGHT, Z_WEIGHT = 0.01, 0.001                      # of the two losses


# ---- cases --------------------------------------------------------------------------------------------------

def listed():
    return [
        # the experts' inner rows of one decoding step (128 tokens, top-8)
        dict(name="rows4_step", op="rows4", rows=1024, cols=2048, kind="mxfp4"),
        # the same of a prefill chunk (16384 tokens, top-8), with a row scale
        dict(name="rows4_prefill", op="rows4", rows=131072, cols=2048, kind="nvfp4"),
        # hidden states of a prefill batch before dispatch; a width whose scales do not fill 16 bytes
        dict(name="rows4_hidden", op="rows4", rows=16411, cols=7200, kind="mxfp4"),
        # a single request on one rank's 32 experts: eight of them are read
        dict(name="matmul4_one_token", op="matmul4", tokens=1, experts=32, topk=8, inner=7168, channels=4096, gated=True,
             kind="mxfp4", routing="uniform"),
        # a decoding step of 128 requests, gate and up projections: bound by the weights
        dict(name="matmul4_step", op="matmul4", tokens=128, experts=32, topk=8, inner=7168, channels=4096, gated=True,
             kind="mxfp4", routing="uniform"),
        # a prefill chunk: bound by the products
        dict(name="matmul4_prefill", op="matmul4", tokens=2048, experts=32, topk=8, inner=7168, channels=4096, gated=True,
             kind="mxfp4", routing="uniform"),
        # the second projection of that chunk
        dict(name="matmul4_down", op="matmul4", tokens=2048, experts=32, topk=8, inner=2048, channels=7168, gated=False,
             kind="nvfp4", routing="uniform"),
        # skewed routing, odd sizes
        dict(name="matmul4_ragged", op="matmul4", tokens=1237, experts=60, topk=6, inner=1440, channels=2040, gated=False,
             kind="nvfp4", routing="zipf"),
        # a small batch of 4 ranks x 96 tokens, one of them half empty (latency only)
        dict(name="balance_small", op="balance", ranks=4, tokens=96, experts=60, topk=4, score="softmax", per_rank=True,
             logits="float32", ragged=True, add=False),
        # a training batch of 32 ranks x 512 tokens: bf16 logits, the gradient of the gate weights added
        dict(name="balance_train", op="balance", ranks=32, tokens=512, experts=128, topk=8, score="softmax", per_rank=False,
             logits="bfloat16", ragged=False, add=True),
        # 16 ranks x 4096 tokens, normalised sigmoid scores, a loss for each rank's sequence
        dict(name="balance_large", op="balance", ranks=16, tokens=4096, experts=256, topk=8, score="sigmoid", per_rank=True,
             logits="float32", ragged=True, add=False),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rows4", "matmul4", "matmul4", "balance"])
    kind = rng.choice(["mxfp4", "nvfp4"])
    if op == "rows4":
        cols = rng.choice([1024, 2048, 4096, 7168, 32 * rng.randint(4, 250)])
        return dict(op=op, rows=min(_spread(rng, 1, 131072), (1 << 28) // cols), cols=cols, kind=kind)
    if op == "balance":
        ranks = rng.choice([1, 2, 4, 8, 16, 32])
        per_rank = _spread(rng, 1, 65536 // ranks)
        experts = rng.choice([e for e in (8, 16, 60, 64, 96, 128, 160, 256, 384) if e % ranks == 0])
        return dict(op=op, ranks=ranks, tokens=min(per_rank, 65536 * 256 // experts // ranks), experts=experts,
                    topk=rng.randint(1, min(8, experts)), score=rng.choice(["softmax", "sigmoid"]),
                    per_rank=rng.random() < 0.5, logits=rng.choice(["float32", "bfloat16"]),
                    ragged=rng.random() < 0.5, add=rng.random() < 0.5)
    experts = rng.choice([8, 16, 24, 32, 60])
    inner = 32 * _spread(rng, 8, 224)
    channels = 2 * _spread(rng, 64, 3584)
    while experts * inner * channels > 32 * 7168 * 4096:
        channels = 2 * (channels // 4)
    topk = rng.randint(1, 8)
    return dict(op=op, tokens=_spread(rng, 1, 16384 // topk), experts=experts, topk=topk, inner=inner,
                channels=channels, gated=rng.random() < 0.5, kind=kind, routing=rng.choice(["uniform", "zipf"]))


def work(case):
    if case["op"] == "rows4":                               # bf16 in, the codes' values in bf16 out
        n, c = case["rows"], case["cols"]
        return {"bytes": 4 * n * c + (4 * n if case["kind"] == "nvfp4" else 0), "flops": 4 * n * c}
    if case["op"] == "balance":
        n, e = case["ranks"] * case["tokens"], case["experts"]
        size = 4 if case["logits"] == "float32" else 2
        groups = case["ranks"] if case["per_rank"] else 1
        return {"bytes": n * (e * size * (3 if case["add"] else 2) + 4 * case["topk"]) + groups * e * 8, "flops": 10 * n * e}
    e, k, t = case["experts"], case["topk"], case["tokens"]
    rows, inner, n = t * k, case["inner"], case["channels"]
    busy = e if case["routing"] == "uniform" and t * k > 8 * e else min(e, rows)
    if t == 1:
        busy = k
    wide = n // 2 if case["gated"] else n
    row = inner // 2 + inner // BLOCK[case["kind"]] + (4 if case["kind"] == "nvfp4" else 0)
    return {"bytes": rows * (row + 2 * wide) + busy * n * row, "flops": 2 * rows * inner * n}


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
        _contexts[key] = binding.MoEContext(R, T, H, E, K, allow_unrouted=True)
    return _contexts[key]


def _routing(t, e, k, routing, g):
    """Distinct experts for every token: the k largest of e random keys, even or with Zipf popularity."""
    keys = -torch.log(torch.rand((t, e), generator=g, device=DEV).clamp_(1e-9, 1 - 1e-7))
    if routing == "zipf":                                   # exponential races: the smallest arrival times win
        order = torch.argsort(torch.rand(e, generator=g, device=DEV)).to(torch.float32)
        keys = keys * (order + 1.0) ** 1.2
    return torch.argsort(keys, dim=1)[:, :k].to(torch.int32).contiguous()


def _random_codes(g, rows, cols):
    """Packed codes of normal values in units of their scales, the first of a pair in the low half."""
    v = _normal(g, rows, cols).mul_(2.0)
    mid = torch.tensor(MIDPOINTS, device=DEV)
    code = torch.bucketize(v.abs(), mid).to(torch.uint8) + (v < 0).to(torch.uint8) * 8
    return code[:, 0::2] + code[:, 1::2] * 16


def _random_scales(g, rows, cols, kind, level):
    """Block scales [rows, cols / block] around 2^level in rows of whole 16 bytes, and the scales of rows (nvfp4)."""
    n = cols // BLOCK[kind]
    buf = torch.zeros((rows, (n + 15) // 16 * 16), dtype=torch.uint8, device=DEV)
    if kind == "mxfp4":
        buf[:, :n] = torch.randint(126 + level, 129 + level, (rows, n), generator=g, device=DEV).to(torch.uint8)
        return buf.view(SCALE_TYPE[kind])[:, :n], None
    unit = torch.rand((rows, n), generator=g, device=DEV).add_(0.5).mul_(64.0)
    buf[:, :n] = unit.to(torch.float8_e4m3fn).view(torch.uint8)
    rows_scale = (0.5 + torch.rand(rows, generator=g, device=DEV)) * 2.0 ** (level - 6)
    return buf.view(SCALE_TYPE[kind])[:, :n], rows_scale


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"] == "rows4":
        n, c = case["rows"], case["cols"]
        s["x"] = _normal(g, n, c).mul_(0.5 + torch.rand((n, 1), generator=g, device=DEV)).to(torch.bfloat16)
        if own:
            from paper_2607_26444_b200 import binding
            s["ctx"] = _context(1, 1, 8, 1, 1)
            s["rows4"] = binding.empty_rows4((n,), c, case["kind"])
            s["y"] = torch.empty((n, c), dtype=torch.bfloat16, device=DEV)
    elif case["op"] == "matmul4":
        e, inner, n, kind = case["experts"], case["inner"], case["channels"], case["kind"]
        rows = case["tokens"] * case["topk"]
        ids = _routing(case["tokens"], e, case["topk"], case["routing"], g)
        s["counts"] = torch.bincount(ids.reshape(-1).long(), minlength=e).tolist()
        s["a"] = _random_codes(g, rows, inner)
        s["a_block"], s["a_scale"] = _random_scales(g, rows, inner, kind, -1)
        s["w"] = torch.empty((e, n, inner // 2), dtype=torch.uint8, device=DEV)
        for i in range(e):
            s["w"][i] = _random_codes(g, n, inner)
        block, scale = _random_scales(g, e * n, inner, kind, -1 - int(round(math.log2(inner) / 2)))
        s["w_block"] = block.unflatten(0, (e, n))
        s["w_scale"] = None if scale is None else scale.view(e, n)
        if own:
            s["ctx"] = _context(1, case["tokens"], 8, e, case["topk"])
            s["layout"] = s["ctx"].layout(ids)
            s["out"] = torch.empty((rows, n // 2 if case["gated"] else n), dtype=torch.bfloat16, device=DEV)
    else:
        r, t, e, k = case["ranks"], case["tokens"], case["experts"], case["topk"]
        popular = _normal(g, e).mul_(0.7)                   # the imbalance that the loss is there to remove
        s["logits"] = (_normal(g, r, t, e) + popular).to(getattr(torch, case["logits"]))
        keys = s["logits"].float().view(r * t, e) + 0.1 * _normal(g, r * t, e)
        s["ids"] = torch.argsort(keys, dim=1, descending=True)[:, :k].to(torch.int32).view(r, t, k).contiguous()
        if case["ragged"]:                                  # tokens behind a rank's last one are padding
            used = torch.randint((t + 1) // 2, t + 1, (r, 1), generator=g, device=DEV)
            s["ids"].masked_fill_((torch.arange(t, device=DEV) >= used)[:, :, None], -1)
        groups = r if case["per_rank"] else 1
        if case["add"]:
            s["add"] = _normal(g, r, t, e).mul_(0.01 / (r * t)).to(s["logits"].dtype)
        if own:
            from paper_2607_26444_b200 import binding
            s["ctx"] = _context(r, t, 8, e, k)
            s["params"] = binding.make_balance(case["score"], weight=WEIGHT, z_weight=Z_WEIGHT, per_rank=case["per_rank"])
            s["stats"] = s["ctx"].balance_stats(s["params"])
            s["loss"] = torch.empty(2, dtype=torch.float32, device=DEV)
            s["dlogits"] = torch.empty_like(s["logits"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    if case["op"] == "rows4":
        ctx.quantize_rows4(s["x"], s["rows4"])
        ctx.dequantize_rows4(s["rows4"], s["y"])
        return {"y": s["y"]} if case["kind"] == "mxfp4" else {"y": s["y"], "scale": s["rows4"].scale}
    if case["op"] == "matmul4":
        from paper_2607_26444_b200 import binding
        ctx.expert_matmul4(s["layout"], binding.Rows4(s["a"], s["a_block"], s["a_scale"]),
                           binding.Rows4(s["w"], s["w_block"], s["w_scale"]), s["out"], gated=case["gated"])
        return {"y": s["out"]}
    ctx.balance_loss(s["params"], s["logits"], s["ids"], s["loss"], s["stats"])
    ctx.balance_grad(s["params"], s["logits"], s["ids"], s["stats"], s["dlogits"], add=s.get("add"))
    return {"loss": s["loss"], "count": s["stats"].count, "prob": s["stats"].prob, "dlogits": s["dlogits"]}


def _run_plain(s):
    op = s["case"]["op"]
    return _plain_rows4(s) if op == "rows4" else _plain_matmul4(s) if op == "matmul4" else _plain_balance(s)


def _nearest_code(u):
    """Values of the nearest e2m1 codes, ties to the even code; beyond 6 the largest."""
    a = u.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.where(u < 0, -1.0, 1.0) * (torch.round(a / step) * step).clamp(max=6.0)


def _plain_rows4(s):
    kind = s["case"]["kind"]
    x = s["x"].float()
    blocks = x.view(x.shape[0], -1, BLOCK[kind])
    top = blocks.abs().amax(dim=2, keepdim=True)
    if kind == "mxfp4":
        exponent = torch.frexp(top).exponent - 3            # 2^(exponent + 2) <= top
        exponent = exponent + (top >= torch.ldexp(torch.full_like(top, 7.0), exponent)).to(exponent.dtype)
        scale = torch.ldexp(torch.ones_like(top), exponent.clamp(min=-126))
        return {"y": (_nearest_code(blocks / scale) * scale).view(x.shape).to(torch.bfloat16)}
    # both quotients have exact numerators and denominators: what lies between two codes is seen as such
    row = x.abs().amax(dim=1)[:, None, None]
    block = (448.0 * top / torch.where(row == 0, 1.0, row)).to(torch.float8_e4m3fn).float()
    unit = row * block
    q = _nearest_code(2688.0 * blocks / torch.where(unit == 0, 1.0, unit)) * (unit != 0)
    scale = row / 2688.0
    return {"y": (q * (block * scale)).view(x.shape).to(torch.bfloat16), "scale": scale.flatten()}


def _values(codes, block, kind):
    """What packed codes [n, cols / 2] and their block scales stand for."""
    table = torch.tensor(CODE_VALUES + [-v for v in CODE_VALUES], device=DEV)
    pairs = torch.stack((codes & 15, codes >> 4), dim=2).flatten(1)
    v = table[pairs.int()].unflatten(1, (-1, BLOCK[kind]))
    return (v * block.float()[:, :, None]).flatten(1)


def _plain_matmul4(s):
    """Expert by expert: rows times weights, the scales of rows and channels, the gate."""
    case = s["case"]
    n, kind = case["channels"], case["kind"]
    a = _values(s["a"], s["a_block"], kind)
    y = torch.empty((a.shape[0], n // 2 if case["gated"] else n), dtype=torch.float32, device=DEV)
    first = 0
    for e, count in enumerate(s["counts"]):
        if count:
            r = slice(first, first + count)
            p = a[r] @ _values(s["w"][e], s["w_block"][e], kind).t()
            if s["a_scale"] is not None:
                p = p * s["a_scale"][r, None] * s["w_scale"][e]
            y[r] = p[:, :n // 2] / (1.0 + torch.exp(-p[:, :n // 2])) * p[:, n // 2:] if case["gated"] else p
            first += count
    return {"y": y.to(torch.bfloat16)}


def _plain_balance(s):
    case = s["case"]
    r, t, e, k = case["ranks"], case["tokens"], case["experts"], case["topk"]
    groups = r if case["per_rank"] else 1
    l = s["logits"].float().view(groups, -1, e)
    ids = s["ids"].view(groups, -1, k)
    routed = (ids >= 0).any(dim=2, keepdim=True).float()    # padding tokens take no part
    m = l.amax(dim=2, keepdim=True)
    ex = torch.exp(l - m)
    total = ex.sum(dim=2, keepdim=True)
    soft, lse = ex / total, m + torch.log(total)
    if case["score"] == "softmax":
        p, slope = soft, 1.0
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
        p = score / score.sum(dim=2, keepdim=True)
        slope = 1.0 / (1.0 + torch.exp(l))                  # of the logarithm of the score
    n = routed.sum(dim=1)                                   # [groups, 1]
    slots = ids.reshape(groups, -1)
    count = torch.zeros((groups, e), device=DEV).scatter_add_(1, slots.clamp(min=0).long(), (slots >= 0).float())
    safe = n.clamp(min=1.0)
    prob = (p * routed).sum(dim=1) / safe
    alive = (n > 0).float().sum().clamp(min=1.0)
    f = count * e / (k * safe)
    loss = WEIGHT * (f * prob).sum() / alive
    z = Z_WEIGHT * (lse * lse * routed).sum() / n.sum().clamp(min=1.0)
    c = (WEIGHT / alive * f / safe)[:, None]
    d = p * slope * (c - (p * c).sum(dim=2, keepdim=True))
    d = (d + 2.0 * Z_WEIGHT / n.sum().clamp(min=1.0) * lse * soft) * routed
    d = d.view(s["logits"].shape)
    if case["add"]:
        d = d + s["add"].float()
    return {"loss": torch.stack((loss, z)), "count": count.to(torch.int32), "prob": prob, "dlogits": d.to(s["logits"].dtype)}


# ---- the definition in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    with_own = globals()["own"]
    globals()["own"] = False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = with_own
    return {"rows4": _exact_rows4, "matmul4": _exact_matmul4, "balance": _exact_balance}[case["op"]](s)


def _decoded(packed, block, scale):
    """Values in 64 bits from the bits: a code is sign, two exponent bits and one fraction bit."""
    n = packed.shape[0]
    code = torch.empty((n, packed.shape[1] * 2), dtype=torch.uint8, device=DEV)
    code[:, 0::2], code[:, 1::2] = packed % 16, packed // 16
    power, half = (code // 2 % 4).double(), (code % 2).double()
    v = torch.where(power == 0, half / 2, (1 + half / 2) * torch.exp2(power - 1)) * (1 - 2 * (code // 8).double())
    bits = block.contiguous().view(torch.uint8).double()
    if scale is None:
        unit = torch.exp2(bits - 127)
    else:
        power, part = torch.floor(bits / 8), bits % 8
        unit = torch.where(power == 0, part * 2.0 ** -9, (1 + part / 8) * torch.exp2(power - 7)) * scale.double()[:, None]
    return v * unit.repeat_interleave(v.shape[1] // unit.shape[1], dim=1)


def _exact_matmul4(s):
    n = s["case"]["channels"]
    first, out = 0, []
    for e, count in enumerate(s["counts"]):
        if count == 0:
            continue
        r = slice(first, first + count)
        first += count
        flat = s["a_scale"] is None
        a = _decoded(s["a"][r], s["a_block"][r], None if flat else s["a_scale"][r])
        w = _decoded(s["w"][e], s["w_block"][e], None if flat else s["w_scale"][e])
        y = torch.einsum("rk,ck->rc", a, w)
        out.append(torch.nn.functional.silu(y[:, :n // 2]) * y[:, n // 2:] if s["case"]["gated"] else y)
    return {"y": torch.cat(out)}


def _exact_codes(u):
    """The nearest of the eight magnitudes by its neighbours' midpoints; on a midpoint the even code."""
    mid = torch.tensor(MIDPOINTS, dtype=torch.float64, device=DEV)
    a = u.abs().contiguous()
    below, upto = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    code = torch.where(below % 2 == 0, below, upto)
    return torch.tensor(CODE_VALUES, dtype=torch.float64, device=DEV)[code] * u.sign()


def _exact_rows4(s):
    kind = s["case"]["kind"]
    out, scales = [], []
    for x in s["x"].split(8192):                            # 64 bits of everything at once would not fit
        b = x.double().unflatten(1, (-1, BLOCK[kind]))
        top = b.abs().amax(2, keepdim=True)
        if kind == "mxfp4":
            low = torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2
            scale = torch.exp2(torch.where(top < 7 * torch.exp2(low), low, low + 1))
            out.append((_exact_codes(b / scale) * scale).flatten(1))
            continue
        row = x.double().abs().amax(1)
        scales.append(row / 2688)
        row = row[:, None, None]
        block = torch.where(row == 0, 0.0, 448 * top / row).float().to(torch.float8_e4m3fn).double()
        code = _exact_codes(torch.where(block == 0, 0.0, 2688 * b / (row * block)))
        out.append((code * block * row / 2688).flatten(1))
    y = torch.cat(out)
    return {"y": y} if kind == "mxfp4" else {"y": y, "scale": torch.cat(scales)}


def _exact_balance(s):
    case = s["case"]
    r, e, k = case["ranks"], case["experts"], case["topk"]
    logits = s["logits"].double().requires_grad_()
    losses, squares, counts, probs, tokens = [], [], [], [], 0
    parts = zip(logits, s["ids"]) if case["per_rank"] else [(logits.flatten(0, 1), s["ids"].flatten(0, 1))]
    for l, ids in parts:
        keep = (ids >= 0).any(1)
        l, chosen = l[keep], ids[keep]
        n = l.shape[0]
        counts.append(torch.bincount(chosen[chosen >= 0].long(), minlength=e))
        if n == 0:
            probs.append(torch.zeros(e, dtype=torch.float64, device=DEV))
            continue
        score = torch.softmax(l, 1) if case["score"] == "softmax" else torch.sigmoid(l)
        mean = (score / score.sum(1, keepdim=True)).mean(0)
        probs.append(mean.detach())
        losses.append((mean * counts[-1]).sum() * e / (k * n))
        squares.append(torch.logsumexp(l, 1).square().sum())
        tokens += n
    loss = torch.stack((WEIGHT * torch.stack(losses).mean(), Z_WEIGHT * torch.stack(squares).sum() / tokens))
    loss.sum().backward()
    d = logits.grad + s["add"].double() if case["add"] else logits.grad
    return {"loss": loss.detach(), "count": torch.stack(counts).to(torch.int32), "prob": torch.stack(probs), "dlogits": d}
