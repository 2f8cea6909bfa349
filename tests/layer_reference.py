"""The operators of include/strata_layer.h in 64 bits, written from their formulas with numpy, for the tests."""
import numpy as np

CODE_MAX = {"int8": 127.0, "e4m3": 448.0}


def bf16(a):
    """Nearest bf16 (ties to even) of float64 values, as float64.  Finite values only."""
    a = np.asarray(a, dtype=np.float64)
    m, e = np.frexp(a)                                  # a = m * 2^e, 0.5 <= |m| < 1: 8 significant bits
    return np.ldexp(np.rint(m * 256.0), e - 8)


def route_scores(logits, score):
    """Scores [n, E]; NaN and -inf logits score zero."""
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-l))
    m = l.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        t = np.where(l == m, 1.0, np.exp(l - m))
    t = np.where(l == -np.inf, 0.0, t)
    total = t.sum(axis=1, keepdims=True)
    return t / np.where(total == 0, 1.0, total)


def route_choice(logits, score, bias, n_group, topk_group, group_score, dtype=np.float64):
    """Choice values [n, E] after the group stage; -inf = not to be chosen."""
    s = route_scores(logits, score)
    dead = np.isnan(logits) | (logits == -np.inf)
    by_sum = n_group > 1 and group_score == "top2"
    c = (s + (0.0 if bias is None else bias.astype(np.float64))) if bias is not None or by_sum else logits.astype(np.float64)
    c = np.where(dead | np.isnan(c), -np.inf, c)
    if n_group > 1:
        n, E = c.shape
        g = np.sort(c.reshape(n, n_group, E // n_group), axis=2)[:, :, ::-1]
        best = g[:, :, 0].copy()
        if by_sum and E // n_group > 1:
            best += np.where(np.isinf(g[:, :, 1]), 0.0, g[:, :, 1])
        order = np.argsort(-best, axis=1, kind="stable")[:, :topk_group]
        keep = np.zeros((n, n_group), bool)
        np.put_along_axis(keep, order, True, axis=1)
        keep &= best > -np.inf
        c = np.where(np.repeat(keep, E // n_group, axis=1), c, -np.inf)
    return c


def route_ids(choice, k):
    ids = np.argsort(-choice, axis=1, kind="stable")[:, :k]
    return np.where(np.take_along_axis(choice, ids, 1) > -np.inf, ids, -1)


def route_weights(logits, ids, score, renorm, scale):
    s = route_scores(logits, score)
    w = np.where(ids >= 0, np.take_along_axis(s, np.maximum(ids, 0), 1), 0.0)
    if renorm:
        d = w.sum(axis=1, keepdims=True)
        w = w / np.where(d == 0, 1.0, d)
    return w * scale


def route_grad(logits, ids, dw, score, renorm, scale):
    n, E = logits.shape
    s = route_scores(logits, score)
    dead = np.isnan(logits) | (logits == -np.inf)
    live = (ids >= 0) & ~np.take_along_axis(dead, np.maximum(ids, 0), 1)
    sk = np.where(live, np.take_along_axis(s, np.maximum(ids, 0), 1), 0.0)
    dk = np.where(live, scale * dw.astype(np.float64), 0.0)
    if renorm:
        d = sk.sum(axis=1, keepdims=True)
        safe = np.where(d == 0, 1.0, d)
        dk = np.where(live & (d > 0), (dk - (dk * sk).sum(1, keepdims=True) / safe) / safe, 0.0)
    full = np.zeros((n, E))
    for r in range(n):
        np.add.at(full[r], ids[r][live[r]], dk[r][live[r]])
    if score == "sigmoid":
        g = full * s * (1.0 - s)
    else:
        g = s * (full - (full * s).sum(1, keepdims=True))
    return np.where(dead, 0.0, g)


def norm(h, weight, eps):
    h = h.astype(np.float64)
    return h * weight.astype(np.float64) / np.sqrt((h * h).mean(1, keepdims=True) + eps)


def norm_grad(dy, h, weight, eps, dresidual=None):
    dy, h, weight = dy.astype(np.float64), h.astype(np.float64), weight.astype(np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    hat, g = h * rstd, dy * weight
    dx = rstd * (g - hat * (g * hat).mean(1, keepdims=True))
    return dx if dresidual is None else dx + dresidual.astype(np.float64), (dy * hat).sum(0)


def products(a, w, a_scale, w_scale, offset, count, gated):
    """(out, magnitude): rows outside the segments are NaN; magnitude = sum |a w| scaled, for error bounds."""
    rows, channels = a.shape[0], w.shape[1]
    y = np.full((rows, channels), np.nan)
    mag = np.full((rows, channels), np.nan)
    for e in range(w.shape[0]):
        r = slice(int(offset[e]), int(offset[e]) + int(count[e]))
        scale = a_scale[r].astype(np.float64)[:, None] * w_scale[e].astype(np.float64)[None]
        y[r] = (a[r].astype(np.float64) @ w[e].astype(np.float64).T) * scale
        mag[r] = (np.abs(a[r].astype(np.float64)) @ np.abs(w[e].astype(np.float64)).T) * scale
    if not gated:
        return y, mag, None
    g, u = y[:, :channels // 2], y[:, channels // 2:]
    gm, um = mag[:, :channels // 2], mag[:, channels // 2:]
    with np.errstate(over="ignore"):
        s = g / (1.0 + np.exp(-g))
    # |d silu| <= 1.1, so an error of x in the gate moves the product by 1.1 * x * |up|
    return s * u, 1.1 * gm * np.abs(u) + np.abs(s) * um, g
