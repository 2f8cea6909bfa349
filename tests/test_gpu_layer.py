"""The operators of include/strata_layer.h on the GPU against plain 64-bit implementations (layer_reference.py).

Tolerances, derived before the first run (u = 2^-24, the unit roundoff of binary32):
- ids: the order of the 64-bit choice values, where two of them differ by more than their binary32 rounding; exact
  ties go to the lower index;
- gate weights: an exponential (2 ulp, and its argument's rounding, u * |l - m|), a sum of E/32 + 5 or K terms and two
  divisions: relative 2u * (E/32 + 5 + K + 8 + max|l|);
- bf16 results: half an ulp (8 significant bits: 2^-8 of the value's power of two), plus a few binary32 roundings
  (2^-18 relative of the terms);
- 8-bit codes of the quantiser: bit-exact against the correctly rounded binary32 quotient; those of the norm: half a step
  around the 64-bit value (1 + 2^-10 for the binary32 value's own error);
- int8 products are exact sums, scaled: half a bf16 ulp + 2^-18 relative; e4m3 products are summed by the matrix unit in binary32
  storage with at least 13 fraction bits kept in each alignment: 2^-13 * sum|a w|;
- dweight: n terms in binary32 in some fixed order: (n + 8) * u * sum|dy hat|."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2607_26444_b200 import binding as B

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import layer_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def half_ulp(a):
    """Half a bf16 ulp at every value."""
    return np.ldexp(1.0, np.frexp(a)[1] - 9)                   # |a| = m * 2^e with 0.5 <= m < 1: an ulp is 2^(e - 8)


def strided(t, extra):
    """The same values in rows that are `extra` elements further apart; the gap holds a sentinel."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), 77.0, device=t.device).to(t.dtype)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


# ---- router --------------------------------------------------------------------------------------------------

ROUTES = [
    dict(n=1, E=256, K=8, score="sigmoid", bias=True, G=8, kg=4, gs="top2", renorm=True, scale=2.5, dt=torch.float32),
    dict(n=37, E=256, K=8, score="sigmoid", bias=True, G=8, kg=4, gs="top2", renorm=True, scale=2.5, dt=torch.float32),
    dict(n=300, E=128, K=8, score="softmax", bias=False, G=1, kg=1, gs="max", renorm=False, scale=1.0, dt=torch.bfloat16),
    dict(n=65, E=60, K=4, score="softmax", bias=False, G=4, kg=2, gs="max", renorm=True, scale=1.0, dt=torch.float32),
    dict(n=33, E=60, K=6, score="sigmoid", bias=True, G=6, kg=3, gs="top2", renorm=False, scale=1.5, dt=torch.float32),
    dict(n=40, E=160, K=6, score="softmax", bias=False, G=8, kg=3, gs="max", renorm=False, scale=16.0, dt=torch.float32),
    dict(n=17, E=384, K=8, score="sigmoid", bias=True, G=8, kg=5, gs="max", renorm=True, scale=1.0, dt=torch.bfloat16),
    dict(n=19, E=8, K=8, score="softmax", bias=True, G=1, kg=1, gs="max", renorm=True, scale=1.0, dt=torch.float32),
    dict(n=9, E=1, K=1, score="softmax", bias=False, G=1, kg=1, gs="max", renorm=False, scale=1.0, dt=torch.float32),
    dict(n=12, E=1024, K=32, score="softmax", bias=False, G=32, kg=32, gs="top2", renorm=True, scale=1.0, dt=torch.float32),
    dict(n=12, E=1000, K=32, score="sigmoid", bias=False, G=1, kg=1, gs="max", renorm=True, scale=1.0, dt=torch.float32),
    dict(n=14, E=31, K=3, score="sigmoid", bias=True, G=1, kg=1, gs="max", renorm=True, scale=1.0, dt=torch.bfloat16),
    dict(n=21, E=64, K=7, score="softmax", bias=True, G=32, kg=9, gs="top2", renorm=False, scale=1.0, dt=torch.float32),
    # more tokens than resident warps: a warp decides several, and up to eight slots two at a time
    dict(n=9777, E=256, K=8, score="sigmoid", bias=True, G=8, kg=4, gs="top2", renorm=True, scale=2.5, dt=torch.float32),
    dict(n=14211, E=64, K=6, score="softmax", bias=False, G=1, kg=1, gs="max", renorm=False, scale=1.0, dt=torch.bfloat16),
    dict(n=5001, E=60, K=5, score="softmax", bias=False, G=6, kg=2, gs="max", renorm=True, scale=1.0, dt=torch.float32),
    dict(n=5003, E=384, K=10, score="sigmoid", bias=True, G=8, kg=4, gs="max", renorm=False, scale=1.0, dt=torch.float32),
]


def route_case(c, extra=0, seed=3):
    g = gen(seed)
    logits = (randn(g, c["n"], c["E"]) * 2).to(c["dt"])
    if extra:
        logits = strided(logits, extra)
    bias = randn(g, c["E"]) * 0.1 if c["bias"] else None
    ctx = B.MoEContext(1, c["n"], 8, c["E"], c["K"])
    params = B.make_route(c["score"], c["renorm"], c["scale"], c["G"], c["kg"], c["gs"])
    ids = torch.full((c["n"], c["K"]), -7, dtype=torch.int32, device=DEV)
    w = torch.full((c["n"], c["K"]), float("nan"), device=DEV)
    return ctx, params, logits, bias, ids, w


def weight_bound(c, logits):
    return 2 * U * (c["E"] / 32 + 5 + c["K"] + 8 + 2 * float(np.abs(logits[np.isfinite(logits)]).max()))


def check_route(c, logits, bias, ids, w):
    l64, b64 = f64(logits), None if bias is None else f64(bias)
    choice = ref.route_choice(l64, c["score"], b64, c["G"], c["kg"], c["gs"])
    got, want = ids.cpu().numpy(), ref.route_ids(choice, c["K"])
    # a different id is accepted only where the two choice values are closer than binary32 resolves
    gc = np.take_along_axis(np.where(np.isinf(choice), -1e30, choice), np.maximum(got, 0), 1)
    wc = np.take_along_axis(np.where(np.isinf(choice), -1e30, choice), np.maximum(want, 0), 1)
    close = np.abs(gc - wc) <= 8 * U * np.maximum(1.0, np.abs(wc))
    assert np.all((got == want) | ((got >= 0) & (want >= 0) & close))
    assert (got != want).mean() < 0.01
    assert all(len(set(r[r >= 0])) == (r >= 0).sum() for r in got)
    ww = ref.route_weights(l64, got, c["score"], c["renorm"], c["scale"])
    np.testing.assert_allclose(f64(w), ww, rtol=weight_bound(c, l64), atol=1e-37)


@pytest.mark.parametrize("c", ROUTES, ids=lambda c: f"{c['n']}x{c['E']}k{c['K']}{c['score']}g{c['G']}")
@pytest.mark.parametrize("extra", [0, 3, 8])
def test_route_against_64_bits(c, extra):
    ctx, params, logits, bias, ids, w = route_case(c, extra)
    ctx.route(params, logits, ids, w, bias=bias)
    assert ctx.device_status() == B.STRATA_OK
    check_route(c, logits, bias, ids, w)


def test_route_ties_go_to_the_lower_index():
    # all equal (more equal keys than one warp holds), then two plateaus
    for E, K in ((256, 8), (1024, 32), (40, 5)):
        ctx = B.MoEContext(1, 3, 8, E, K)
        logits = torch.zeros((3, E), device=DEV)
        logits[1, E // 2:] = 1.0
        logits[2, ::2] = -0.0
        ids = torch.empty((3, K), dtype=torch.int32, device=DEV)
        w = torch.empty((3, K), device=DEV)
        for score in ("softmax", "sigmoid"):
            for bias in (None, torch.zeros(E, device=DEV)):
                ctx.route(B.make_route(score), logits, ids, w, bias=bias)
                got = ids.cpu().numpy()
                assert got[0].tolist() == list(range(K)) and got[1].tolist() == list(range(E // 2, E // 2 + K))
                assert got[2].tolist() == list(range(K))
                np.testing.assert_allclose(f64(w), 1.0 / K, rtol=1e-6)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("groups", [(1, 1, "max"), (8, 4, "top2")])
def test_route_masked_logits(score, bias, groups):
    """Rows with -inf, the lowest finite value, NaN and +inf; a row with fewer than K experts left and one with none."""
    E, K = 64, 8
    inf = float("inf")
    logits = randn(gen(5), 8, E)
    logits[0, :] = -inf
    logits[1, 3:] = -inf                                       # three experts left
    logits[2, ::2] = float("nan")
    logits[3, 5] = inf
    logits[4, :] = torch.finfo(torch.float32).min
    logits[5, 1:] = torch.finfo(torch.float32).min
    logits[6, 10] = inf
    logits[6, 20] = inf
    b = torch.zeros(E, device=DEV) if bias else None
    if bias:
        b[7] = -inf                                            # an expert taken out by its bias
    G, kg, gs = groups
    ctx = B.MoEContext(1, 8, 8, E, K)
    ids = torch.empty((8, K), dtype=torch.int32, device=DEV)
    w = torch.empty((8, K), device=DEV)
    ctx.route(B.make_route(score, True, 1.0, G, kg, gs), logits, ids, w, bias=b)
    got, gw = ids.cpu().numpy(), f64(w)
    assert np.all(got[0] == -1) and np.all(gw[0] == 0)
    assert set(got[1]) == {0, 1, 2, -1} and np.all(got[1][3:] == -1) and np.all(gw[1][3:] == 0)
    assert abs(gw[1].sum() - 1) < 1e-6
    assert np.all(got[2] % 2 == 1)
    assert got[3][0] == 5 and got[6][:2].tolist() == [10, 20]
    assert np.all(np.isfinite(gw)) and np.all(gw >= 0)
    if score == "softmax":
        assert gw[3][0] == 1.0 and gw[6][0] == gw[6][1] == 0.5
        if not bias:
            np.testing.assert_allclose(gw[4], 1.0 / K, rtol=1e-6)
    if score == "sigmoid":
        assert np.all(gw[4] == 0)                              # every score underflows: no weight to share
    if bias:
        assert 7 not in got[got >= 0]


def test_route_many_tokens_with_ties_and_masks():
    """Tokens that the shorter way decides and tokens that the exact one must (ties, masks, NaN) side by side in one warp."""
    n, E, K = 9500, 128, 8
    g = gen(51)
    logits = (randn(g, n, E) * 4).round() / 4                    # few distinct values: ties everywhere
    logits[::7] = randn(g, logits[::7].shape[0], E)
    logits[3::11, ::2] = -float("inf")
    logits[5::13] = 0.0
    logits[6::17, 40] = float("nan")
    ctx = B.MoEContext(1, n, 8, E, K)
    for score, groups in (("softmax", (1, 1, "max")), ("sigmoid", (4, 2, "top2"))):
        bias = None if score == "softmax" else torch.zeros(E, device=DEV)
        ids = torch.empty((n, K), dtype=torch.int32, device=DEV)
        w = torch.empty((n, K), device=DEV)
        ctx.route(B.make_route(score, True, 1.0, *groups), logits, ids, w, bias=bias)
        l64 = f64(logits)
        # equal logits have equal binary32 scores: the order of the 64-bit scores, rounded, is the order to expect
        choice = ref.route_choice(l64, score, None if bias is None else f64(bias), *groups)
        if score == "softmax":
            assert np.array_equal(ids.cpu().numpy(), ref.route_ids(choice, K))
        else:
            got, want = ids.cpu().numpy(), ref.route_ids(choice, K)
            rows = [i for i in range(n) if i % 7 != 0]             # quarter steps: groups' sums are apart or equal
            assert (got[rows] != want[rows]).mean() < 1e-3
        ww = ref.route_weights(l64, ids.cpu().numpy(), score, True, 1.0)
        np.testing.assert_allclose(f64(w), ww, rtol=2 * U * (E / 32 + 5 + K + 8 + 40), atol=1e-37)


def test_route_ids_feed_the_layout():
    """Unrouted slots (-1) of the router are what the layout skips."""
    ctx = B.MoEContext(2, 8, 8, 16, 4, allow_unrouted=True)
    logits = randn(gen(6), 16, 16)
    logits[3] = -float("inf")
    logits[9, 2:] = -float("inf")
    ids = torch.empty((2, 8, 4), dtype=torch.int32, device=DEV)
    w = torch.empty((2, 8, 4), device=DEV)
    ctx.route(B.make_route(), logits.view(2, 8, 16), ids, w)
    lay = ctx.layout(ids)
    assert ctx.device_status() == B.STRATA_OK
    assert int(lay.expert_count.sum()) == 16 * 4 - 4 - 2


@pytest.mark.parametrize("c", ROUTES, ids=lambda c: f"{c['n']}x{c['E']}k{c['K']}{c['score']}g{c['G']}")
@pytest.mark.parametrize("extra", [0, 3])
def test_route_grad_against_64_bits(c, extra):
    ctx, params, logits, bias, ids, w = route_case(c, extra, seed=11)
    ctx.route(params, logits, ids, w, bias=bias)
    dw = randn(gen(12), c["n"], c["K"])
    ids[0, -1] = -1                                            # a slot that was dropped
    if c["K"] > 2:
        ids[-1, 1] = ids[-1, 0]                                # a repeated expert adds up
    grad = strided(torch.zeros_like(logits), extra) if extra else torch.empty_like(logits)
    ctx.route_grad(params, logits, ids, dw, grad)
    assert ctx.device_status() == B.STRATA_OK
    got = f64(grad)
    i64, l64 = ids.cpu().numpy().astype(np.int64), f64(logits)
    want = ref.route_grad(l64, i64, f64(dw), c["score"], c["renorm"], c["scale"])
    # terms of size scale * max|dw| enter with the relative error of a weight; bf16 results round once more
    tol = 4 * weight_bound(c, l64) * c["scale"] * float(dw.abs().max())
    assert np.all(np.abs(got - want) <= tol + (half_ulp(want) if c["dt"] == torch.bfloat16 else 8 * U * np.abs(want)))
    if extra:
        assert float(grad.as_strided((c["n"], extra), grad.stride(), grad.storage_offset() + c["E"]).float().min()) == 77.0


def test_route_grad_against_differences():
    """Central differences of the forward pass's weights in 64 bits, through the reference that it is tested against."""
    c = dict(n=6, E=16, K=4, score="softmax", renorm=True, scale=1.5)
    for c["score"] in ("softmax", "sigmoid"):
        for c["renorm"] in (True, False):
            g = gen(21)
            logits = randn(g, c["n"], c["E"])
            ctx = B.MoEContext(1, c["n"], 8, c["E"], c["K"])
            params = B.make_route(c["score"], c["renorm"], c["scale"])
            ids = torch.empty((c["n"], c["K"]), dtype=torch.int32, device=DEV)
            w = torch.empty((c["n"], c["K"]), device=DEV)
            ctx.route(params, logits, ids, w)
            dw = randn(g, c["n"], c["K"])
            grad = torch.empty_like(logits)
            ctx.route_grad(params, logits, ids, dw, grad)
            l, i, d, step = f64(logits), ids.cpu().numpy().astype(np.int64), f64(dw), 1e-5
            diff = np.zeros_like(l)
            for e in range(c["E"]):
                hi, lo = l.copy(), l.copy()
                hi[:, e] += step
                lo[:, e] -= step
                diff[:, e] = ((ref.route_weights(hi, i, c["score"], c["renorm"], c["scale"])
                               - ref.route_weights(lo, i, c["score"], c["renorm"], c["scale"])) * d).sum(1) / (2 * step)
            # truncation step^2 and cancellation 1e-16 / step of the differences, binary32 of the gradient
            np.testing.assert_allclose(f64(grad), diff, rtol=1e-5, atol=1e-5)


def test_route_grad_skips_what_it_must():
    E, K = 32, 4
    logits = randn(gen(31), 4, E)
    logits[0, 5] = -float("inf")
    logits[1, :] = -float("inf")
    ids = torch.tensor([[5, 1, 2, 3], [0, 1, 2, 3], [-1, -1, -1, -1], [1, 99, 2, -5]], dtype=torch.int32, device=DEV)
    dw = torch.ones((4, K), device=DEV) * torch.arange(1, K + 1, device=DEV)
    ctx = B.MoEContext(1, 4, 8, E, K)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            grad = torch.full_like(logits, float("nan"))
            ctx.route_grad(B.make_route(score, renorm), logits, ids, dw, grad)
            got = f64(grad)
            assert np.all(np.isfinite(got)) and got[0, 5] == 0 and np.all(got[1] == 0) and np.all(got[2] == 0)
            assert got[3, 1] != 0
            assert ctx.device_status() == B.STRATA_ERR_BAD_EXPERT_ID
    assert ctx.device_status() == B.STRATA_OK


# ---- norm and quantiser ------------------------------------------------------------------------------------------

SHAPES = [(1, 8), (1, 7168), (3, 1000), (5, 1024), (7, 1032), (130, 4096), (300, 2048), (2, 8200), (33, 16384), (3, 32768),
          (4000, 64), (2500, 1544)]
# more rows than the GPU holds at once, of one warp, of part of a block, of a block, of the longest kinds; rows fetched ahead
RING_SHAPES = [(9001, 64), (6003, 1024), (7000, 1544), (1501, 7168), (701, 16384), (401, 32768), (2049, 8712), (2048, 16648)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("out", ["bf16", "int8", "e4m3", "both"])
def test_norm_against_64_bits(rows, cols, residual, out):
    g = gen(rows * 7 + cols)
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    x = strided(randn(g, rows, cols).to(torch.bfloat16), 8)
    weight = 1 + 0.2 * randn(g, cols)
    weight = weight.to(torch.bfloat16) if rows % 2 else weight
    res = (3 * randn(g, rows, cols)).to(torch.bfloat16) if residual else None
    h = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV) if residual else None
    kind = {"bf16": None, "both": "e4m3"}.get(out, out)
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV) if out in ("bf16", "both") else None
    buf = torch.full((rows, cols + B.STRATA_Q8_TRAILER), 0x55, dtype=torch.uint8, device=DEV)
    q, scale = B.q8_rows(buf, CODES[kind]) if kind else (None, None)
    ctx.norm(x, weight, 1e-6, out=y, residual=res, residual_out=h, q=q, q_scale=scale)
    stored = f64(x)
    if residual:
        full = f64(x) + f64(res)                               # exact in 64 bits; binary32 rounds it once before bf16 does
        assert np.all(np.abs(f64(h) - full) <= half_ulp(full) + 2 * U * np.abs(full))
        stored = f64(h)
    want = ref.norm(stored, f64(weight), 1e-6)
    err = 2.0 ** -18 * np.abs(want)
    if y is not None:
        assert np.all(np.abs(f64(y) - want) <= half_ulp(want) + err)
    if kind:
        top = np.abs(want).max(1)
        np.testing.assert_allclose(f64(scale), top / ref.CODE_MAX[kind], rtol=2.0 ** -18)
        s = f64(scale)[:, None]
        value = f64(q) * s
        half = 0.5 * s if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s)
        assert np.all(np.abs(value - want) <= half * (1 + 2.0 ** -10) + err)
        assert np.abs(f64(q)).max() == ref.CODE_MAX[kind]
        assert bool((buf[:, cols + 4:] == 0x55).all())         # only the codes and the scale of a row are written


@pytest.mark.parametrize("rows,cols", RING_SHAPES)
@pytest.mark.parametrize("residual,out", [(False, "bf16"), (True, "both"), (True, "int8")])
def test_norm_of_many_rows_against_64_bits(rows, cols, residual, out):
    test_norm_against_64_bits(rows, cols, residual, out)


def ieee_codes(x, kind):
    """The quantiser's definition: scale = max / limit, codes of the correctly rounded binary32 quotient x * limit / max."""
    x = x.astype(np.float32)
    top = np.abs(x).max(1)
    scale = (top / np.float32(ref.CODE_MAX[kind])).astype(np.float32)
    # exact product and one division in 64 bits: far enough beyond binary32 to round as the quotient itself
    units = (x.astype(np.float64) * ref.CODE_MAX[kind] / np.where(top == 0, 1, top)[:, None].astype(np.float64)).astype(np.float32)
    if kind == "int8":
        return np.rint(units).astype(np.int8).view(np.uint8), scale
    return torch.from_numpy(np.clip(units, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), scale


@pytest.mark.parametrize("rows,cols", SHAPES + RING_SHAPES)
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_quantize_rows_bit_exact(rows, cols, kind):
    g = gen(rows + cols)
    x = (randn(g, rows, cols) * (10.0 ** (6 * torch.rand((rows, 1), generator=g, device=DEV) - 3))).to(torch.bfloat16)
    x[rows // 2] = 0
    x[0, cols // 2] = -abs(float(x[0].float().abs().max())) * 2        # the largest magnitude is negative
    x = strided(x, 16)
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    q = torch.empty((rows, cols), dtype=CODES[kind], device=DEV)
    scale = torch.empty(rows, device=DEV)
    ctx.quantize_rows(x, q, scale)
    codes, s = ieee_codes(x.float().cpu().numpy(), kind)
    assert np.array_equal(scale.cpu().numpy().view(np.uint32), s.view(np.uint32))
    got = q.view(torch.uint8).cpu().numpy()
    if kind == "e4m3":                                                   # -0 and +0 are the same value
        got, codes = np.where(got == 0x80, 0, got), np.where(codes == 0x80, 0, codes)
    assert np.array_equal(got, codes)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("top", [2.0 ** -130, 2.0 ** -126, 2.0 ** -118, 3.0e38])
def test_quantize_rows_extreme_scales(kind, top):
    """Rows whose scale is subnormal or near the largest binary32: the division, not a reciprocal, decides."""
    cols = 264
    x = (torch.linspace(-1, 1, cols, device=DEV)[None] * top).to(torch.bfloat16)
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    q = torch.empty((1, cols), dtype=CODES[kind], device=DEV)
    scale = torch.empty(1, device=DEV)
    ctx.quantize_rows(x, q, scale)
    codes, s = ieee_codes(x.float().cpu().numpy(), kind)
    assert np.array_equal(scale.cpu().numpy().view(np.uint32), s.view(np.uint32))
    got = q.view(torch.uint8).cpu().numpy()
    assert np.array_equal(np.where(got == 0x80, 0, got), np.where(codes == 0x80, 0, codes))


def test_norm_in_place_zero_rows_and_streams():
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    g = gen(2)
    x, r = randn(g, 50, 512).to(torch.bfloat16), randn(g, 50, 512).to(torch.bfloat16)
    w = torch.ones(512, device=DEV)
    apart_h, apart_y = torch.empty_like(x), torch.empty_like(x)
    ctx.norm(x, w, 1e-5, out=apart_y, residual=r, residual_out=apart_h)
    x2, r2 = x.clone(), r.clone()
    ctx.norm(x2, w, 1e-5, out=x2, residual=r2, residual_out=r2)          # out = x, residual_out = residual
    assert torch.equal(x2, apart_y) and torch.equal(r2, apart_h)
    ctx.norm(x[:0], w, 1e-5, out=apart_y[:0])                              # no rows
    zero = torch.zeros((2, 512), dtype=torch.bfloat16, device=DEV)
    y, q, s = torch.empty_like(zero), torch.empty((2, 512), dtype=torch.int8, device=DEV), torch.empty(2, device=DEV)
    ctx.norm(zero, w, 1e-5, out=y, q=q, q_scale=s)
    assert not y.any() and not q.any() and not s.any()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        big = torch.empty_like(x)
        ctx.norm(x, w, 1e-5, out=big)
    side.synchronize()
    want = ref.norm(f64(x), f64(w), 1e-5)
    assert np.all(np.abs(f64(big) - want) <= half_ulp(want) + 2.0 ** -18 * np.abs(want))


@pytest.mark.parametrize("rows,cols", SHAPES + RING_SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_grad_against_64_bits(rows, cols, residual):
    g = gen(rows * 3 + cols)
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    h = strided((2 * randn(g, rows, cols)).to(torch.bfloat16), 8)
    dy = randn(g, rows, cols).to(torch.bfloat16)
    weight = 1 + 0.2 * randn(g, cols)
    weight = weight if rows % 2 else weight.to(torch.bfloat16)
    dres = strided(randn(g, rows, cols).to(torch.bfloat16), 24) if residual else None
    dx = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    dw = torch.full((cols,), float("nan"), device=DEV)
    ctx.norm_grad(dy, h, weight, 1e-6, dx, dw, dresidual=dres)
    want, dwant = ref.norm_grad(f64(dy), f64(h), f64(weight), 1e-6, None if dres is None else f64(dres))
    h64, dy64 = f64(h), f64(dy)
    rstd = 1 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-6)
    gg = np.abs(dy64 * f64(weight))
    terms = rstd * (gg + np.abs(h64 * rstd) * (gg * np.abs(h64 * rstd)).mean(1, keepdims=True))
    terms = terms + (np.abs(f64(dres)) if residual else 0)
    assert np.all(np.abs(f64(dx) - want) <= half_ulp(want) + 2.0 ** -18 * terms)
    mag = np.abs(dy64 * h64 * rstd).sum(0)
    assert np.all(np.abs(f64(dw) - dwant) <= (rows + 8) * U * mag + 8 * U * np.abs(dwant))
    again = torch.empty_like(dw)
    ctx.norm_grad(dy, h, weight, 1e-6, dx, again, dresidual=dres)
    assert torch.equal(dw, again)                                          # the order of the sum is fixed


def test_norm_grad_against_differences():
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    g = gen(9)
    h, dy, w = randn(g, 3, 16).to(torch.bfloat16), randn(g, 3, 16).to(torch.bfloat16), 1 + 0.1 * randn(g, 16)
    dx, dw = torch.empty_like(h), torch.empty(16, device=DEV)
    ctx.norm_grad(dy, h, w, 1e-3, dx, dw)
    h64, dy64, w64, step = f64(h), f64(dy), f64(w), 1e-5
    for c in range(16):
        for array, got in ((h64, None), (w64, None)):
            hi, lo = array.copy(), array.copy()
            hi[..., c] += step
            lo[..., c] -= step
            if array is h64:
                d = ((ref.norm(hi, w64, 1e-3) - ref.norm(lo, w64, 1e-3)) * dy64).sum(1) / (2 * step)
                np.testing.assert_allclose(f64(dx)[:, c], d, rtol=2.0 ** -8, atol=1e-4)
            else:
                d = ((ref.norm(h64, hi, 1e-3) - ref.norm(h64, lo, 1e-3)) * dy64).sum() / (2 * step)
                np.testing.assert_allclose(f64(dw)[c], d, rtol=1e-5, atol=1e-5)


def test_norm_grad_in_place_and_no_rows():
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    g = gen(10)
    h, dy, r = (randn(g, 40, 256).to(torch.bfloat16) for _ in range(3))
    w = torch.ones(256, device=DEV)
    dx, dw = torch.empty_like(h), torch.empty(256, device=DEV)
    ctx.norm_grad(dy, h, w, 1e-6, dx, dw, dresidual=r)
    for target in (dy, r):
        d2, r2 = dy.clone(), r.clone()
        out = d2 if target is dy else r2
        ctx.norm_grad(d2, h, w, 1e-6, out, torch.empty_like(dw), dresidual=r2)
        assert torch.equal(out, dx)
    ctx.norm_grad(dy[:0], h[:0], w, 1e-6, dx[:0], dw)
    assert not dw.any()


# ---- the experts' products --------------------------------------------------------------------------------------------

def matmul_case(tokens, E, K, inner, channels, gated, kind, seed, R=1, skew=False, pad=0, **ctx_kw):
    g = gen(seed)
    ctx = B.MoEContext(R, tokens, 8, E, K, **ctx_kw)
    if skew:                                                       # most tokens want the first experts; some get none
        keys = torch.rand((R * tokens, E), generator=g, device=DEV) * (1 + torch.arange(E, device=DEV)) ** 2
    else:
        keys = torch.rand((R * tokens, E), generator=g, device=DEV)
    ids = torch.argsort(keys, dim=1)[:, :K].to(torch.int32).reshape(R, tokens, K).contiguous()
    if ctx_kw.get("allow_unrouted"):
        ids[:, ::3] = -1
    lay = ctx.layout(ids)
    rows = ctx.recv_rows

    def codes(*shape):
        v = randn(g, *shape)
        if kind == "int8":
            return (v * 40).round().clamp(-127, 127).to(torch.int8)
        return (v * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    a = torch.zeros((rows, inner + pad), dtype=CODES[kind], device=DEV)
    a[:, :inner] = codes(rows, inner)
    a = a[:, :inner]
    w = codes(E, channels, inner)
    a_scale = (0.5 + torch.rand(rows, generator=g, device=DEV)) / 40
    w_scale = (0.5 + torch.rand((E, channels), generator=g, device=DEV)) / (40 * inner ** 0.5)
    out = torch.full((rows, channels // 2 if gated else channels), 99.0, dtype=torch.bfloat16, device=DEV)
    return ctx, lay, a, a_scale, w, w_scale, out


def check_products(lay, a, a_scale, w, w_scale, out, gated, kind, count=None):
    count = lay.expert_count.cpu().numpy() if count is None else count
    want, mag, gate = ref.products(f64(a), f64(w), f64(a_scale), f64(w_scale), lay.expert_offset.cpu().numpy(), count, gated)
    got = f64(out)
    used = ~np.isnan(want[:, 0])
    assert np.all(got[~used] == 99.0)                              # rows of no segment are not written
    got, want, mag = got[used], want[used], mag[used]
    rel = 2.0 ** -18 * (1 + (np.abs(gate[used]) if gated else 0))
    sums = 2.0 ** -18 if kind == "int8" else 2.0 ** -13            # gated: the error of each factor meets the other
    bound = half_ulp(want) + rel * np.abs(want) + (sums * mag if gated or kind == "e4m3" else 0) + 1e-30
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], np.argwhere(bad)[:4])


MATMULS = [
    dict(tokens=1, E=8, K=1, inner=16, channels=4),                   # one row, the least of everything
    dict(tokens=1, E=32, K=8, inner=512, channels=256),               # one token
    dict(tokens=5, E=4, K=2, inner=144, channels=100),                # odd sizes below one tile
    dict(tokens=64, E=4, K=2, inner=256, channels=128),
    dict(tokens=100, E=3, K=3, inner=400, channels=132),              # 100 rows each
    dict(tokens=257, E=3, K=2, inner=1040, channels=260, skew=True),  # more than one row tile
    dict(tokens=700, E=7, K=2, inner=272, channels=388, skew=True),   # several row tiles, idle experts
    dict(tokens=33, E=300, K=4, inner=128, channels=64),              # more experts than SMs, most nearly empty
    dict(tokens=900, E=2, K=2, inner=128, channels=1028),
    dict(tokens=40, E=6, K=2, inner=256, channels=640, R=2, segment_align=16),
    dict(tokens=50, E=6, K=2, inner=256, channels=384, allow_unrouted=True),
    dict(tokens=2048, E=2, K=1, inner=64, channels=512),              # short inner extent, many tiles per CTA
    dict(tokens=3000, E=4, K=4, inner=32, channels=1200, skew=True),
    dict(tokens=45, E=5, K=2, inner=160, channels=274),               # an odd number of gated channels: rows of out on two bytes
    dict(tokens=300, E=3, K=2, inner=368, channels=510),
]


@pytest.mark.parametrize("c", MATMULS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_expert_matmul_against_64_bits(c, gated, kind):
    ctx, lay, a, a_scale, w, w_scale, out = matmul_case(gated=gated, kind=kind, seed=41, pad=32, **c)
    ctx.expert_matmul(lay, a, a_scale, w, w_scale, out, gated=gated)
    assert ctx.device_status() == B.STRATA_OK
    check_products(lay, a, a_scale, w, w_scale, out, gated, kind)
    first = out.clone()
    ctx.expert_matmul(lay, a, a_scale, w, w_scale, out, gated=gated)
    assert torch.equal(first, out)


@pytest.mark.parametrize("gated", [False, True])
def test_expert_matmul_fixed_capacity(gated):
    ctx, lay, a, a_scale, w, w_scale, out = matmul_case(24, 4, 2, 128, 64, gated, "int8", 5, R=2, slot_capacity=40)
    ctx.expert_matmul(lay, a, a_scale, w, w_scale, out, gated=gated)
    assert ctx.device_status() == B.STRATA_OK
    check_products(lay, a, a_scale, w, w_scale, out, gated, "int8", count=np.full(4, 80))


def test_expert_matmul_odd_channels_and_odd_strides():
    for channels, stride in ((131, 131), (1, 1), (128, 129)):
        ctx, lay, a, a_scale, w, w_scale, out = matmul_case(90, 3, 2, 128, channels, False, "int8", 23)
        wide = torch.full((a.shape[0], stride), 99.0, dtype=torch.bfloat16, device=DEV)
        out = wide[:, :channels]
        ctx.expert_matmul(lay, a, a_scale, w, w_scale, out)
        check_products(lay, a, a_scale, w, w_scale, out, False, "int8")
        assert bool((wide[:, channels:] == 99.0).all())


def test_expert_matmul_extreme_codes_are_exact():
    """All codes at +-127 over the longest inner extent: the int32 sums come near their limit and stay exact."""
    inner = 131056
    ctx, lay, a, a_scale, w, w_scale, out = matmul_case(3, 2, 2, inner, 4, False, "int8", 8)
    a.fill_(127)
    w.fill_(127)
    w[:, 1] = -127
    ctx.expert_matmul(lay, a, a_scale, w, w_scale, out)
    check_products(lay, a, a_scale, w, w_scale, out, False, "int8")


def test_expert_matmul_zero_scales_and_strides():
    ctx, lay, a, a_scale, w, w_scale, out = matmul_case(70, 3, 2, 192, 96, True, "int8", 17)
    a_scale[5] = 0
    w_scale[1, 7] = 0
    rows = a.shape[0]
    wide_scale = torch.zeros((rows, 3), device=DEV)
    wide_scale[:, 0] = a_scale
    wide = torch.full((rows, 48 + 6), 99.0, dtype=torch.bfloat16, device=DEV)
    ctx.expert_matmul(lay, a, wide_scale[:, 0], w, w_scale, wide[:, :48], gated=True)
    check_products(lay, a, a_scale, w, w_scale, wide[:, :48], True, "int8")
    assert bool((wide[:, 48:] == 99.0).all())


# ---- the operators together -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_layer_from_hidden_states_to_output(kind):
    """norm -> router -> layout -> dispatch of 8-bit rows -> gated product -> quantiser -> product -> combine, each stage
    checked on the data of the one before it."""
    R, T, H, E, K, I = 2, 40, 256, 8, 3, 160
    g = gen(77)
    ctx = B.MoEContext(R, T, H, E, K, dispatch_dtype=B.STRATA_Q8_ROW)
    x, res = (randn(g, R, T, H).to(torch.bfloat16) for _ in range(2))
    weight, router = 1 + 0.1 * randn(g, H), randn(g, E, H) / H ** 0.5
    h, y = torch.empty_like(x), torch.empty_like(x)
    sent = torch.zeros((R, T, H + B.STRATA_Q8_TRAILER), dtype=torch.uint8, device=DEV)
    q, q_scale = B.q8_rows(sent, CODES[kind])
    ctx.norm(x, weight, 1e-6, out=y, residual=res, residual_out=h, q=q, q_scale=q_scale)
    ids = torch.empty((R, T, K), dtype=torch.int32, device=DEV)
    gate = torch.empty((R, T, K), device=DEV)
    ctx.route(B.make_route("sigmoid"), y.float() @ router.t(), ids, gate, bias=torch.zeros(E, device=DEV))
    lay = ctx.layout(ids)
    recv = torch.zeros((ctx.recv_rows, H + B.STRATA_Q8_TRAILER), dtype=torch.uint8, device=DEV)
    ctx.register(recv)
    ctx.dispatch(lay, sent, recv)
    src = lay.src_of_row.long() // K
    assert torch.equal(recv, sent.reshape(R * T, -1)[src])          # rows travel bit for bit, scales with them
    a, a_scale = B.q8_rows(recv, CODES[kind])

    def weights(channels, inner):
        v = randn(g, E, channels, inner)
        w = (v * 30).round().clamp(-127, 127).to(torch.int8) if kind == "int8" else (v * 30).to(torch.float8_e4m3fn)
        return w, torch.full((E, channels), 1 / (30 * inner ** 0.5), device=DEV)
    w1, s1 = weights(2 * I, H)
    w2, s2 = weights(H, I)
    mid = torch.full((ctx.recv_rows, I), 99.0, dtype=torch.bfloat16, device=DEV)
    ctx.expert_matmul(lay, a, a_scale, w1, s1, mid, gated=True)
    check_products(lay, a, a_scale, w1, s1, mid, True, kind)
    mq = torch.zeros((ctx.recv_rows, I), dtype=CODES[kind], device=DEV)
    ms = torch.zeros(ctx.recv_rows, device=DEV)
    ctx.quantize_rows(mid, mq, ms, layout=lay)
    codes, s = ieee_codes(mid.float().cpu().numpy(), kind)
    assert np.array_equal(np.where(codes == 0x80, 0, codes), np.where(mq.view(torch.uint8).cpu().numpy() == 0x80, 0, mq.view(torch.uint8).cpu().numpy()))
    back = torch.full((ctx.recv_rows, H), 99.0, dtype=torch.bfloat16, device=DEV)
    ctx.expert_matmul(lay, mq, ms, w2, s2, back)
    check_products(lay, mq, ms, w2, s2, back, False, kind)
    out = torch.empty_like(x)
    ctx.combine(lay, back, gate, out)
    assert ctx.device_status() == B.STRATA_OK
    rows = lay.dst_row.long().reshape(R * T, K)
    want = (f64(back)[rows.cpu().numpy()] * f64(gate).reshape(R * T, K, 1)).sum(1)
    mag = (np.abs(f64(back)[rows.cpu().numpy()]) * f64(gate).reshape(R * T, K, 1)).sum(1)
    assert np.all(np.abs(f64(out).reshape(R * T, H) - want) <= half_ulp(want) + 8 * U * mag)


def test_quantize_rows_stops_at_the_rows_in_use():
    ctx, lay, a, a_scale, w, w_scale, out = matmul_case(30, 6, 2, 64, 64, False, "int8", 3, R=2, segment_align=16)
    x = randn(gen(4), ctx.recv_rows, 64).to(torch.bfloat16)
    q = torch.full((ctx.recv_rows, 64), 55, dtype=torch.int8, device=DEV)
    s = torch.full((ctx.recv_rows,), 55.0, device=DEV)
    ctx.quantize_rows(x, q, s, layout=lay)
    used = int(lay.expert_offset[-1])
    assert used < ctx.recv_rows
    assert bool((q[used:] == 55).all()) and bool((s[used:] == 55).all()) and bool((s[:used] != 55).all())


def test_layer_operators_in_a_cuda_graph():
    """Captured once, replayed on new inputs: nothing of a call's data stays with the host."""
    n, H, E, K, C = 24, 256, 8, 2, 64
    ctx = B.MoEContext(1, n, H, E, K, dispatch_dtype=B.STRATA_Q8_ROW)
    x, weight = torch.empty((n, H), dtype=torch.bfloat16, device=DEV), torch.ones(H, device=DEV)
    logits = torch.empty((n, E), device=DEV)
    sent = torch.zeros((n, H + B.STRATA_Q8_TRAILER), dtype=torch.uint8, device=DEV)
    recv = torch.zeros((n * K, H + B.STRATA_Q8_TRAILER), dtype=torch.uint8, device=DEV)
    ctx.register(recv)
    q, qs = B.q8_rows(sent, torch.int8)
    a, a_s = B.q8_rows(recv, torch.int8)
    ids, w = torch.empty((n, K), dtype=torch.int32, device=DEV), torch.empty((n, K), device=DEV)
    g = gen(15)
    wt = (randn(g, E, C, H) * 30).round().clamp(-127, 127).to(torch.int8)
    ws = torch.full((E, C), 1 / (30 * 16.0), device=DEV)
    out = torch.full((n * K, C), 99.0, dtype=torch.bfloat16, device=DEV)
    lay, params = ctx.new_layout(), B.make_route()

    def step():
        ctx.norm(x, weight, 1e-6, q=q, q_scale=qs)
        ctx.route(params, logits, ids, w)
        ctx.layout(ids, lay)
        ctx.dispatch(lay, sent, recv)
        ctx.expert_matmul(lay, a, a_s, wt, ws, out)
    x.copy_(randn(g, n, H))
    logits.copy_(randn(g, n, E))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        x.copy_(randn(g, n, H) * (k + 1))
        logits.copy_(randn(g, n, E))
        graph.replay()
        torch.cuda.synchronize()
        check_products(lay, a, a_s, wt, ws, out, False, "int8")
        assert torch.equal(recv, sent[lay.src_of_row.long() // K])
    assert ctx.device_status() == B.STRATA_OK
