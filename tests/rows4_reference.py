"""4-bit rows and the balance loss in 64 bits, written from their formulas with numpy, for the tests."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = {"mxfp4": 32, "nvfp4": 16}


def code_of(u):
    """Magnitude codes (0..7) nearest to |u|; half-way cases to the even code."""
    mid = (VALUES[1:] + VALUES[:-1]) / 2
    a = np.abs(u)
    low, high = np.searchsorted(mid, a, side="left"), np.searchsorted(mid, a, side="right")
    return np.where(low % 2 == 0, low, high)


def e4m3_table():
    b = np.arange(127, dtype=np.float64)                      # 0x00 .. 0x7e, finite and increasing
    e, m = np.floor(b / 8), b % 8
    return np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7))


def e4m3_of(v):
    """Codes nearest to v >= 0, half-way cases to the even code."""
    table = e4m3_table()
    mid = (table[1:] + table[:-1]) / 2
    low, high = np.searchsorted(mid, v, side="left"), np.searchsorted(mid, v, side="right")
    return np.where(low % 2 == 0, low, high).astype(np.uint8)


def block_values(bits, kind):
    bits = bits.astype(np.int64)
    if kind == "mxfp4":
        return np.where(bits == 255, np.nan, np.ldexp(1.0, bits - 127))
    sign = np.where(bits >= 128, -1.0, 1.0)
    table = np.append(e4m3_table(), np.nan)
    return sign * table[bits & 127]


def quantize(x, kind):
    """(magnitude codes with the sign in bit 3, block scale bytes, row scales) of finite float64 rows."""
    n = BLOCK[kind]
    b = x.reshape(x.shape[0], -1, n)
    top = np.abs(b).max(2)
    if kind == "mxfp4":
        s = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 3, -127)
        s = np.clip(s + ((top >= np.ldexp(7.0, s)) & (top > 0)), -127, 125)
        bits, rows = (s + 127).astype(np.uint8), None
        q = b / np.ldexp(1.0, s)[:, :, None]
    else:
        a = np.abs(x).max(1)[:, None]
        bits = e4m3_of(np.where(a > 0, 448 * top / np.where(a > 0, a, 1.0), 0.0))
        rows = (a[:, 0].astype(np.float32) / np.float32(2688.0)).astype(np.float64)
        unit = (a * block_values(bits, kind))[:, :, None]
        q = np.where(unit > 0, 2688 * b / np.where(unit > 0, unit, 1.0), 0.0)
    codes = code_of(q) + 8 * (np.signbit(b) & (code_of(q) > 0))
    return codes.reshape(x.shape).astype(np.uint8), bits, rows


def unpack(packed):
    """[.., n] bytes -> [.., 2 n] codes; a negative zero is given as zero."""
    c = np.stack((packed & 15, packed >> 4), axis=-1).reshape(*packed.shape[:-1], -1)
    return np.where(c == 8, 0, c)


def values(packed, bits, kind, rows=None):
    c = unpack(packed)
    v = VALUES[c & 7] * np.where(c & 8, -1.0, 1.0)
    unit = block_values(bits, kind)
    if rows is not None:
        unit = unit * rows[..., None]
    return v * np.repeat(unit, BLOCK[kind], axis=-1)


def balance(logits, ids, score, weight, z_weight):
    """Groups [G, n, E], [G, n, K] -> (losses, count, prob, gradient of balance, gradient of z)."""
    G, n, E = logits.shape
    K = ids.shape[2]
    part = ((ids >= 0) & (ids < E)).any(2)
    dead = np.isnan(logits) | (logits == -np.inf)
    l = np.where(dead, -np.inf, logits.astype(np.float64))
    m = np.where(np.isinf(l.max(2, keepdims=True)), 0.0, l.max(2, keepdims=True))
    ex = np.exp(l - m)
    total = ex.sum(2, keepdims=True)
    soft = ex / np.where(total > 0, total, 1.0)
    lse = np.where(total > 0, m + np.log(np.where(total > 0, total, 1.0)), 0.0)
    if score == "softmax":
        p, slope = soft, np.ones_like(soft)
    else:
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-l))
            slope = 1 / (1 + np.exp(l))
        d = s.sum(2, keepdims=True)
        p = s / np.where(d > 0, d, 1.0)
    count = np.zeros((G, E), np.int64)
    for g in range(G):
        k = ids[g][(ids[g] >= 0) & (ids[g] < E)]
        count[g] = np.bincount(k, minlength=E)
    tokens = part.sum(1)
    safe = np.maximum(tokens, 1)[:, None]
    prob = (p * part[:, :, None]).sum(1) / safe
    f = count * E / (K * safe)
    alive, all_tokens = max((tokens > 0).sum(), 1), max(tokens.sum(), 1)
    loss = weight * (f * prob).sum() / alive
    z = z_weight * (lse[:, :, 0] ** 2 * part).sum() / all_tokens
    c = (weight / alive * f / safe)[:, None]
    keep = part[:, :, None] & ~dead
    db = np.where(keep, p * slope * (c - (p * c).sum(2, keepdims=True)), 0.0)
    dz = np.where(keep, 2 * z_weight / all_tokens * lse * soft, 0.0)
    return np.array([loss, z]), count, tokens, prob, db, dz
