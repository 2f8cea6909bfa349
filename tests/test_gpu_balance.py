"""Balance loss, counts and gradient on the GPU against the 64-bit formulas (rows4_reference.balance).

Tolerances, derived before the first run (u = 2^-24):
- a score: an exponential (2 ulp and its argument's rounding, u * |l - max|), a sum of E/32 + 5 terms, a quotient: relative
  s = 2u * (E/32 + 5 + 8 + max|l|); a mean over n tokens adds n/8 + 8 roundings at worst: s + u * (n + 16);
- log-sum-exp: absolute s + 2 ulp of itself; its square twice that;
- losses: the sum over E experts adds E u, the groups G u;
- a gradient entry: the terms p (|c| + sum p |c|) and |z term|, each within 3 s + 8 u, and half a step of the type it is stored in
  (bf16: 2^-8 of the power of two)."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2607_26444_b200 import binding as B

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import rows4_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def case(R, T, E, K, dtype, seed, ragged, extra=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    logits = (2 * torch.randn((R * T, E + extra), generator=g, device=DEV)).to(dtype)[:, :E]
    ids = torch.argsort(torch.rand((R * T, E), generator=g, device=DEV), dim=1)[:, :K].to(torch.int32).reshape(R, T, K).contiguous()
    if ragged:
        used = torch.randint(0, T + 1, (R, 1), generator=g, device=DEV)
        used[-1] = 0                                              # a rank without tokens
        ids.masked_fill_((torch.arange(T, device=DEV) >= used)[:, :, None], -1)
        ids[0, 0, -1] = -1                                        # a token with a dropped slot
    return B.MoEContext(R, T, 8, E, K, allow_unrouted=True), logits, ids


def run(ctx, params, logits, ids, **kw):
    stats = ctx.balance_stats(params)
    loss = torch.full((2,), float("nan"), device=DEV)
    dlogits = torch.full(logits.shape, float("nan"), device=DEV).to(logits.dtype)
    ctx.balance_loss(params, logits, ids, loss, stats)
    ctx.balance_grad(params, logits, ids, stats, dlogits, **kw)
    return loss, stats, dlogits


def check(ctx, params, score, weight, z_weight, logits, ids, loss, stats, dlogits, dloss=(1.0, 1.0), add=None):
    G = ctx.R if params.per_rank else 1
    l64, K, E = f64(logits).reshape(G, -1, ctx.E), ctx.K, ctx.E
    want, count, tokens, prob, db, dz = ref.balance(l64, ids.cpu().numpy().reshape(G, -1, K), score, weight, z_weight)
    finite = np.abs(l64[np.isfinite(l64)])
    s = 2 * U * (E / 32 + 13 + (2 * finite.max() if finite.size else 0))
    n = l64.shape[1]
    assert np.array_equal(stats.count.cpu().numpy(), count) and np.array_equal(stats.tokens.cpu().numpy(), tokens)
    np.testing.assert_allclose(f64(stats.prob), prob, rtol=s + U * (n + 16), atol=1e-37)
    np.testing.assert_allclose(f64(loss)[0], want[0], rtol=s + U * (n + 16 + E + G), atol=1e-37)
    top = finite.max() + np.log(E) if finite.size else 0
    np.testing.assert_allclose(f64(loss)[1], want[1], rtol=U * (n + 32 + G), atol=abs(z_weight) * 2 * top * (s + 2 * U * top))
    c = abs(weight) * count * E / (K * np.maximum(tokens, 1)[:, None] ** 2)
    scale = np.where((tokens > 0)[:, None, None], (3 * s + 16 * U), 0)
    terms = abs(dloss[0]) * scale * np.repeat((c.max(1, keepdims=True) * 2)[:, :, None], E, 2) * np.ones_like(db)
    if score == "softmax":                                        # p times the coefficients
        p = np.exp(np.where(np.isnan(l64), -np.inf, l64) - np.nanmax(np.where(np.isinf(l64), np.nan, l64), axis=2, keepdims=True, initial=-1e30))
        terms = terms * np.minimum(1.0, p)
    d = dloss[0] * db + dloss[1] * dz
    terms = terms + abs(dloss[1]) * np.abs(dz) * (3 * s + 16 * U) + abs(dloss[1] * z_weight) * 2 / max(tokens.sum(), 1) * (s + 2 * U * top)
    if add is not None:
        d = d + f64(add).reshape(d.shape)
        terms = terms + 2 * U * np.abs(f64(add).reshape(d.shape))
    got = f64(dlogits).reshape(d.shape)
    step = np.ldexp(1.0, np.maximum(np.frexp(d)[1], -125) - 9) if logits.dtype == torch.bfloat16 else U * np.abs(d)
    bad = ~(np.abs(got - d) <= terms + step + 1e-40)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], d[bad][:4], terms[bad][:4], np.argwhere(bad)[:4])


CASES = [
    dict(R=1, T=1, E=1, K=1, dtype=torch.float32, ragged=False),
    dict(R=1, T=1, E=8, K=2, dtype=torch.bfloat16, ragged=False),
    dict(R=4, T=33, E=60, K=4, dtype=torch.float32, ragged=True),
    dict(R=2, T=300, E=128, K=8, dtype=torch.bfloat16, ragged=False),
    dict(R=8, T=57, E=256, K=8, dtype=torch.float32, ragged=True),
    dict(R=1, T=5000, E=64, K=6, dtype=torch.float32, ragged=True),
    dict(R=31, T=9, E=31, K=3, dtype=torch.bfloat16, ragged=True),
    dict(R=2, T=40, E=1000, K=32, dtype=torch.float32, ragged=False),
    dict(R=1024, T=3, E=1024, K=2, dtype=torch.bfloat16, ragged=True),
    dict(R=16, T=700, E=384, K=7, dtype=torch.float32, ragged=True),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: f"{c['R']}x{c['T']}x{c['E']}k{c['K']}")
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("per_rank", [False, True])
def test_balance_against_64_bits(c, score, per_rank):
    ctx, logits, ids = case(seed=c["E"], extra=5 if c["T"] % 2 else 8, **c)
    params = B.make_balance(score, weight=0.25, z_weight=0.5, per_rank=per_rank)
    loss, stats, dlogits = run(ctx, params, logits, ids)
    assert ctx.device_status() == B.STRATA_OK
    check(ctx, params, score, 0.25, 0.5, logits, ids, loss, stats, dlogits)
    again = run(ctx, params, logits, ids)                                   # the order of the sums is fixed
    assert torch.equal(loss, again[0]) and torch.equal(stats.prob, again[1].prob) and torch.equal(dlogits, again[2])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("z_weight", [0.0, 0.1])
def test_balance_masked_logits(score, z_weight):
    """NaN and -inf score zero; a token of which nothing is left adds nothing; large logits stay finite."""
    ctx, logits, ids = case(2, 30, 40, 3, torch.float32, 3, False)
    logits[3, ::2] = -float("inf")
    logits[4, 5] = float("nan")
    logits[7] = -float("inf")
    logits[9] = float("nan")
    logits[11] = 80.0 * logits[11]
    params = B.make_balance(score, weight=1.0, z_weight=z_weight)
    loss, stats, dlogits = run(ctx, params, logits, ids)
    check(ctx, params, score, 1.0, z_weight, logits, ids, loss, stats, dlogits)
    assert not dlogits[7].any() and not dlogits[9].any() and float(dlogits[4, 5]) == 0


@pytest.mark.parametrize("shift", [-60.0, -80.0, -95.0, -200.0])
@pytest.mark.parametrize("experts", [40, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_balance_tiny_scores(shift, experts, dtype):
    """Tokens whose sigmoid scores add up to a subnormal number, or to less than binary32 holds, beside ordinary ones: their
    quotients are those of the exponentials (the scores are, within 2^-86 of themselves)."""
    ctx, logits, ids = case(2, 30, experts, 3, dtype, 4, False)
    logits[1::2] += shift
    logits[5, 3:] = -float("inf")
    for z_weight in (0.0, 0.1):
        params = B.make_balance("sigmoid", weight=1.0, z_weight=z_weight)
        loss, stats, dlogits = run(ctx, params, logits, ids)
        check(ctx, params, "sigmoid", 1.0, z_weight, logits, ids, loss, stats, dlogits)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_balance_incoming_gradients(dtype):
    ctx, logits, ids = case(3, 50, 96, 4, dtype, 8, True)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    wide = (0.01 * torch.randn((150, 104), generator=g, device=DEV)).to(dtype)
    add, dloss = wide[:, :96], torch.tensor([2.5, -0.75], device=DEV)
    params = B.make_balance("softmax", weight=0.5, z_weight=0.01, per_rank=True)
    loss, stats, dlogits = run(ctx, params, logits, ids, dloss=dloss, add=add)
    check(ctx, params, "softmax", 0.5, 0.01, logits, ids, loss, stats, dlogits, (2.5, -0.75), add)
    padding = (ids.reshape(150, 4) < 0).all(1)
    assert bool(padding.any()) and torch.equal(dlogits[padding], add[padding])
    wide[:, 96:] = 7.0
    ctx.balance_grad(params, logits, ids, stats, add, dloss=dloss, add=add)                # in place
    assert torch.equal(add, dlogits) and bool((wide[:, 96:] == 7.0).all())


def test_balance_no_tokens_and_bad_ids():
    ctx, logits, ids = case(2, 20, 16, 2, torch.float32, 5, False)
    params = B.make_balance("sigmoid", weight=1.0, z_weight=1.0, per_rank=True)
    ids.fill_(-1)
    loss, stats, dlogits = run(ctx, params, logits, ids)
    assert not loss.any() and not stats.count.any() and not stats.tokens.any() and not stats.prob.any() and not dlogits.any()
    assert ctx.device_status() == B.STRATA_OK
    ids[0, 3] = torch.tensor([16, 1], dtype=torch.int32)
    ids[1, 2] = torch.tensor([-2, 99], dtype=torch.int32)
    loss, stats, dlogits = run(ctx, params, logits, ids)
    assert ctx.device_status() == B.STRATA_ERR_BAD_EXPERT_ID
    check(ctx, params, "sigmoid", 1.0, 1.0, logits, ids, loss, stats, dlogits)


def test_balance_gradient_against_differences():
    for score in ("softmax", "sigmoid"):
        ctx, logits, ids = case(2, 3, 6, 2, torch.float32, 11, False)
        params = B.make_balance(score, weight=1.0, z_weight=0.3, per_rank=True)
        dlogits = run(ctx, params, logits, ids)[2]
        l64, k, step = f64(logits).reshape(2, 3, 6), ids.cpu().numpy(), 1e-5
        for at in np.ndindex(l64.shape):
            hi, lo = l64.copy(), l64.copy()
            hi[at] += step
            lo[at] -= step
            d = (ref.balance(hi, k, score, 1.0, 0.3)[0].sum() - ref.balance(lo, k, score, 1.0, 0.3)[0].sum()) / (2 * step)
            np.testing.assert_allclose(f64(dlogits).reshape(l64.shape)[at], d, rtol=1e-4, atol=1e-6)


def test_balance_captured_and_replayed():
    """Both calls in a CUDA graph on another stream, replayed on new logits and ids."""
    ctx, logits, ids = case(4, 100, 64, 4, torch.bfloat16, 2, True)
    params = B.make_balance("softmax", weight=0.1, z_weight=0.1)
    stats, loss, dlogits = ctx.balance_stats(params), torch.zeros(2, device=DEV), torch.empty_like(logits)

    def step():
        ctx.balance_loss(params, logits, ids, loss, stats)
        ctx.balance_grad(params, logits, ids, stats, dlogits)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    _, other, other_ids = case(4, 100, 64, 4, torch.bfloat16, 77, True)
    logits.copy_(other)
    ids.copy_(other_ids)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    check(ctx, params, "softmax", 0.1, 0.1, logits, ids, loss, stats, dlogits)
