"""Balance loss and gradient on the GPU where they can go wrong: padding beside live tokens, far-apart bf16 logits, long sums of few
experts, and every entry of the gradient.  Tolerances are derived beside each test before its first run (u = 2^-24)."""
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


def make(R, T, E, K, dtype, seed, spread=2.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    logits = (spread * torch.randn((R * T, E), generator=g, device=DEV)).to(dtype)
    ids = torch.argsort(torch.rand((R * T, E), generator=g, device=DEV), dim=1)[:, :K].to(torch.int32).reshape(R, T, K).contiguous()
    return B.MoEContext(R, T, 8, E, K, allow_unrouted=True), logits, ids


def run(ctx, params, logits, ids):
    stats = ctx.balance_stats(params)
    loss, dlogits = torch.empty(2, device=DEV), torch.empty_like(logits)
    ctx.balance_loss(params, logits, ids, loss, stats)
    ctx.balance_grad(params, logits, ids, stats, dlogits)
    assert ctx.device_status() == B.STRATA_OK
    return loss, stats, dlogits


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts", [8, 60, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padding_changes_no_bit(score, experts, dtype):
    """What stands in the logits of padding tokens, which may share a warp with live ones, shows nowhere."""
    ctx, logits, ids = make(2, 51, experts, 4, dtype, experts)
    ids.view(102, 4)[1::2] = -1
    ids.view(102, 4)[70:] = -1
    live = (ids.view(102, 4) >= 0).any(1)
    params = B.make_balance(score, weight=1.0, z_weight=0.1)
    loss, stats, dlogits = run(ctx, params, logits, ids)
    for value in (float("nan"), float("inf"), -float("inf"), 1e4, -1e4):
        other = logits.clone()
        other[~live] = value
        loss2, stats2, dlogits2 = run(ctx, params, other, ids)
        assert torch.equal(loss, loss2) and torch.equal(stats.prob, stats2.prob) and torch.equal(stats.count, stats2.count)
        assert torch.equal(dlogits, dlogits2) and not bool(dlogits2[~live].any())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts", [40, 96, 160, 400])
def test_mean_scores_of_far_apart_bf16_logits(score, experts):
    """One token, so that the mean scores are its scores: they are as exact for bf16 logits as for binary32.

    Logits are multiples of 1/2 from 0 to -80 (bf16 holds them, and their differences are exact).  Roundings of a score, in u: its
    exponential 4 (2 ulp); the exponentials of the sum 4; the sum, 8 or 16 terms in a lane and 5 exchanges, 21; its reciprocal and the product
    2; for a sigmoid a sum (1), a reciprocal within an ulp (2) and a product (1), once for the score and once for the sum, 8.  The
    log-sum-exp is between 0 and 7 and takes the sum's 25 u and 2 ulp of itself; its square twice that, and a rounding."""
    ctx, _, ids = make(1, 1, experts, 3, torch.bfloat16, 1)
    g = torch.Generator().manual_seed(experts)
    logits = (-0.5 * torch.randint(0, 161, (1, experts), generator=g))
    logits[0, torch.randperm(experts, generator=g)[0]] = 0
    logits = logits.to(torch.bfloat16).to(DEV)
    params = B.make_balance(score, weight=1.0, z_weight=1.0)
    loss, stats, _ = run(ctx, params, logits, ids)
    want, _, _, prob, _, _ = ref.balance(f64(logits)[None], ids.cpu().numpy(), score, 1.0, 1.0)
    normal = prob > 2.0 ** -120
    assert normal.sum() > experts // 2
    np.testing.assert_allclose(f64(stats.prob)[normal], prob[normal], rtol=(31 + (8 if score == "sigmoid" else 0)) * U)
    lse = np.sqrt(want[1])
    np.testing.assert_allclose(f64(loss)[1], want[1], rtol=0, atol=2 * lse * (25 + 4 * max(lse, 1)) * U + 2 * U * want[1])


@pytest.mark.parametrize("R,T,E,per_rank,launches", [
    (1, 300, 8, False, 1), (4, 96, 60, True, 1), (1, 1024, 60, False, 1), (1, 2049, 16, False, 2), (1, 16384, 16, False, 2),
    (1, 65537, 8, False, 2), (1, 70000, 4, False, 2), (8, 8192, 8, True, 2), (2, 3000, 128, True, 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_long_sums_of_few_experts(R, T, E, per_rank, launches, score):
    """Many partial sums per expert are added up by a launch of their own, few by the first one's last block.

    A mean score is a sum of positive terms: each within 40 u + 2 u max|l| (a score), added up by at most T / 64 tokens in a run of
    lanes, 64 runs, 19 slices in a lane and 5 exchanges; a division.  A loss adds E and R terms and two roundings of its factors.
    A log-sum-exp (its mean square is above 1) is off by 40 u and 4 u of itself, the mean of its squares twice that and the sums' roundings."""
    ctx, logits, ids = make(R, T, E, min(3, E), torch.float32, E)
    params = B.make_balance(score, weight=0.5, z_weight=0.25, per_rank=per_rank)
    stats, loss = ctx.balance_stats(params), torch.empty(2, device=DEV)
    before = ctx.launch_count()
    ctx.balance_loss(params, logits, ids, loss, stats)
    assert ctx.launch_count() - before == launches
    groups = R if per_rank else 1
    want, count, tokens, prob, _, _ = ref.balance(f64(logits).reshape(groups, -1, E), ids.cpu().numpy().reshape(groups, -1, ctx.K),
                                                  score, 0.5, 0.25)
    assert np.array_equal(stats.count.cpu().numpy(), count) and np.array_equal(stats.tokens.cpu().numpy(), tokens)
    rel = (40 + 2 * float(logits.abs().max()) + T * R / groups / 64 + 90) * U
    np.testing.assert_allclose(f64(stats.prob), prob, rtol=rel)
    np.testing.assert_allclose(f64(loss)[0], want[0], rtol=rel + (E + R + 8) * U)
    np.testing.assert_allclose(f64(loss)[1], want[1], rtol=2 * rel + 16 * U)
    assert ctx.device_status() == B.STRATA_OK


@pytest.mark.parametrize("R,T,E,K,dtype", [
    (1, 3, 8, 2, torch.float32), (4, 33, 60, 4, torch.float32), (2, 300, 128, 8, torch.bfloat16), (8, 57, 256, 8, torch.float32),
    (2, 40, 1000, 32, torch.float32), (16, 700, 384, 7, torch.float32), (4, 50, 500, 5, torch.bfloat16)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("z_weight", [0.0, 0.5])
def test_every_entry_of_the_gradient(R, T, E, K, dtype, score, z_weight):
    """Entry e of a token is p (c - sum p c) times 1 - s for a sigmoid, and 2 z lse softmax / N, so that its error has the factor p too.

    Relative to itself, in u: a score s = 2 (E / 32 + 16 + 2.4 max|l|) (exponentials of 2 ulp, or 2 + 1.2 |l - max| for bf16, arguments'
    roundings, a sum of E / 32 + 5 terms, reciprocals, products); c 8; 1 - s 14 + 4.8 max|l| at most; the product 4.  The sum p c is off by s + E / 32 + 13 of
    sum p |c|; log-sum-exp by s, and 4 of itself.  Half a step of the stored type is 2^-9 of the power of two above (bf16) or u.
    The check itself is checked: zeros, an expectation with the scores of another expert, and one without the factor 1 - s fail it."""
    ctx, logits, ids = make(R, T, E, K, dtype, E + K)
    params = B.make_balance(score, weight=0.25, z_weight=z_weight, per_rank=True)
    got = f64(run(ctx, params, logits, ids)[2]).reshape(R, T, E)
    l = f64(logits).reshape(R, T, E)
    _, count, tokens, _, db, dz = ref.balance(l, ids.cpu().numpy(), score, 0.25, z_weight)
    want, top = db + dz, np.abs(l).max()
    ex = np.exp(l - l.max(2, keepdims=True))
    soft = ex / ex.sum(2, keepdims=True)
    lse = l.max(2, keepdims=True) + np.log(ex.sum(2, keepdims=True))
    p, slope = soft, np.ones_like(soft)
    if score == "sigmoid":
        p = 1 / (1 + np.exp(-l))
        p, slope = p / p.sum(2, keepdims=True), 1 - p
    c = (0.25 / R * count * E / (K * tokens[:, None] ** 2.0))[:, None]
    dot = (p * c).sum(2, keepdims=True)
    s = 2 * (E / 32 + 16 + 2.4 * top)
    tol = p * slope * U * ((s + 8 + 14 + 4.8 * top + 4) * np.abs(c - dot) + 8 * c + (s + E / 32 + 21) * dot)
    tol = tol + 2 * z_weight / tokens.sum() * soft * U * (s + (s + 12) * np.abs(lse))
    step = np.ldexp(1.0, np.maximum(np.frexp(want)[1], -125) - 9) if dtype == torch.bfloat16 else U * np.abs(want)
    tol = tol + step + 1e-40
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4])
    norm = np.linalg.norm
    assert norm(tol) <= (2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -11) * norm(want)
    wrong = [np.zeros_like(want), np.roll(p, 1, axis=2) * slope * (c - dot) + np.roll(dz, 1, axis=2)]
    if score == "sigmoid" and z_weight == 0:                  # beside the z term in bf16 the factor need not show
        wrong.append(p * (c - dot))
    for other in wrong:
        assert (np.abs(got - other) > tol).mean() > 0.75
