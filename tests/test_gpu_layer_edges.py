"""Edges of the layer operators on the GPU.  Helpers and tolerances are those of test_gpu_layer.py."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2607_26444_b200 import binding as B

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import layer_reference as ref  # noqa: E402
import test_gpu_layer as base  # noqa: E402

pytestmark = pytest.mark.gpu
DEV, U = base.DEV, base.U


# ---- router ------------------------------------------------------------------------------------------------------

# Group counts that leave lanes of a warp without a group: a lane would have to hold more than 32 experts.
WIDE_GROUPS = [(960, 3), (800, 5), (800, 20), (594, 9), (561, 17), (1023, 31)]


@pytest.mark.parametrize("n", [7, 5003])
@pytest.mark.parametrize("E,G", WIDE_GROUPS)
@pytest.mark.parametrize("score,bias,gs,renorm", [("sigmoid", True, "top2", True), ("sigmoid", False, "max", True),
                                                  ("softmax", False, "max", False), ("softmax", False, "max", True),
                                                  ("softmax", True, "max", True)])
def test_route_considers_every_expert_of_wide_groups(n, E, G, score, bias, gs, renorm):
    c = dict(n=n, E=E, K=8, score=score, bias=bias, G=G, kg=(G + 1) // 2, gs=gs, renorm=renorm, scale=1.0, dt=torch.float32)
    ctx, params, logits, b, ids, w = base.route_case(c)
    ctx.route(params, logits, ids, w, bias=b)
    assert ctx.device_status() == B.STRATA_OK
    base.check_route(c, logits, b, ids, w)


# Scores whose sum lies below scale / (largest binary32): sigmoid(-88) = 6.05e-39, so scale / sum is infinite and the weights
# are not.  Such a score is subnormal: its rounding is within 2^-150, 2^-22 of the smallest here (2.9e-39); exp(88) adds its
# 2^-23, the sum 1 + exp 2^-24, and the sum of K scores (K - 1) 2^-150 / (K * 2.9e-39) < 2^-22.  A weight is a quotient of two of
# these, rounded twice: 2 * (2^-22 + 2^-23 + 2^-24) + 2^-22 + 2^-23 < 2^-19.
TINY = 2.0 ** -19


@pytest.mark.parametrize("n", [5, 9501])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("K,scale", [(1, 2.5), (8, 64.0), (8, 1.0), (12, 64.0)])
def test_route_weights_of_tiny_scores(n, bias, K, scale):
    E = 64
    logits = torch.full((n, E), -88.5, device=DEV)
    logits += 0.5 * torch.rand((n, E), generator=base.gen(3), device=DEV)
    ctx = B.MoEContext(1, n, 8, E, K)
    ids, w = torch.empty((n, K), dtype=torch.int32, device=DEV), torch.empty((n, K), device=DEV)
    b = torch.rand(E, generator=base.gen(4), device=DEV) if bias else None
    ctx.route(B.make_route("sigmoid", True, scale), logits, ids, w, bias=b)
    got = base.f64(w)
    want = ref.route_weights(base.f64(logits), ids.cpu().numpy(), "sigmoid", True, scale)
    assert np.all(np.isfinite(got))
    np.testing.assert_allclose(got, want, rtol=TINY)


@pytest.mark.parametrize("renorm", [True, False])
def test_route_grad_of_tiny_scores(renorm):
    n, E, K, scale = 40, 64, 8, 2.5
    g = base.gen(5)
    logits = -88.5 + 0.5 * torch.rand((n, E), generator=g, device=DEV)
    ctx = B.MoEContext(1, n, 8, E, K)
    ids = torch.argsort(torch.rand((n, E), generator=g, device=DEV), dim=1)[:, :K].to(torch.int32).contiguous()
    dw = 10 * base.randn(g, n, K)
    grad = torch.empty_like(logits)
    ctx.route_grad(B.make_route("sigmoid", renorm, scale), logits, ids, dw, grad)
    got = base.f64(grad)
    assert np.all(np.isfinite(got))
    want = ref.route_grad(base.f64(logits), ids.cpu().numpy().astype(np.int64), base.f64(dw), "sigmoid", renorm, scale)
    # renormalised: scale * (dw - dot) * weight, terms of scale * max|dw|; otherwise scale * dw * score, subnormal
    size = scale * float(dw.abs().max())
    assert np.all(np.abs(got - want) <= (2 * TINY * size if renorm else TINY * np.abs(want) + size * 2.0 ** -148))


def test_route_grad_of_fp32_logits_keeps_the_exponential_exact():
    """Far below the largest logit too.  Whole logits, so that differences are exact; of the experts that were not chosen, so that
    nothing cancels: -s_e * d * s_k.  Relative error, K = 1: expf within 2 ulp (2^-22) in s_e, s_k and each sum; a sum of E/32
    + 5 terms and its reciprocal, twice; five products: 4 * 2^-22 + (2 * (1 + 5 + 1) + 5) * 2^-24 = 35 u."""
    n, E = 4000, 32
    g = base.gen(8)
    logits = torch.randint(-80, 1, (n, E), generator=g, device=DEV).float()
    logits[:, 0] = 0
    ids = torch.randint(1, E, (n, 1), generator=g, device=DEV).to(torch.int32)
    logits.scatter_(1, ids.long(), -torch.randint(0, 4, (n, 1), generator=g, device=DEV).float())
    dw = torch.ones((n, 1), device=DEV)
    grad = torch.empty_like(logits)
    ctx = B.MoEContext(1, n, 8, E, 1)
    ctx.route_grad(B.make_route("softmax", False), logits, ids, dw, grad)
    i64 = ids.cpu().numpy().astype(np.int64)
    want, got = ref.route_grad(base.f64(logits), i64, base.f64(dw), "softmax", False, 1.0), base.f64(grad)
    np.put_along_axis(want, i64, 1.0, 1)
    np.put_along_axis(got, i64, 1.0, 1)
    np.testing.assert_allclose(got, want, rtol=35 * U)


@pytest.mark.parametrize("n", [6, 9501])
@pytest.mark.parametrize("groups,K", [((1, 1, "max"), 8), ((8, 2, "top2"), 8), ((4, 1, "max"), 3)])
@pytest.mark.parametrize("depth", [90.0, 300.0, 3.0e38])
def test_route_renormalised_softmax_far_below_an_expert_that_is_not_chosen(n, groups, K, depth):
    """The bias chooses experts whose scores are subnormal or zero beside that of the largest logit: their weights are the
    softmax over the chosen logits all the same, and the gradient is that of these weights.  Relative error of a weight as in
    test_gpu_layer.py with |l - max| <= 8: 2 u (K + 8 + 8)."""
    E, scale = 64, 1.5
    g = base.gen(9)
    logits = 4 * torch.rand((n, E), generator=g, device=DEV)
    b = torch.zeros(E, device=DEV)
    b[16:32] = 4.0 + torch.rand(16, generator=g, device=DEV)       # two of the eight groups, one of the four
    logits[:, 16:32] = logits[:, 16:32] - depth                     # at 3e38 all of them are equal
    ctx = B.MoEContext(1, n, 8, E, K)
    params = B.make_route("softmax", True, scale, *groups)
    ids, w = torch.empty((n, K), dtype=torch.int32, device=DEV), torch.empty((n, K), device=DEV)
    ctx.route(params, logits, ids, w, bias=b)
    i64, l64 = ids.cpu().numpy().astype(np.int64), base.f64(logits)
    assert np.all((i64 >= 16) & (i64 < 32))
    chosen = np.take_along_axis(l64, i64, 1)
    t = np.exp(chosen - chosen.max(1, keepdims=True))
    t /= t.sum(1, keepdims=True)
    np.testing.assert_allclose(base.f64(w), scale * t, rtol=2 * U * (K + 16))
    dw, grad = base.randn(g, n, K), torch.empty_like(logits)
    ctx.route_grad(params, logits, ids, dw, grad)
    want = np.zeros((n, E))
    np.put_along_axis(want, i64, scale * t * (base.f64(dw) - (base.f64(dw) * t).sum(1, keepdims=True)), 1)
    assert np.all(np.abs(base.f64(grad) - want) <= 8 * U * (K + 16) * scale * float(dw.abs().max()))


def test_route_of_almost_two_to_the_31_tokens():
    """The strides of warps take the token count past 2^31.  26 to 35 GB in use, a second or two."""
    R, T, E, K = 2, 2 ** 30 - 1, 2, 1
    ctx = B.MoEContext(R, T, 8, E, K)
    n = R * T
    logits = torch.zeros((n, E), dtype=torch.bfloat16, device=DEV)
    logits[::3, 1] = 1.0
    ids = torch.full((n, K), -7, dtype=torch.int32, device=DEV)
    w = torch.full((n, K), -7.0, device=DEV)
    ctx.route(B.make_route("softmax"), logits, ids, w)
    assert ctx.device_status() == B.STRATA_OK
    ones = (n + 2) // 3
    assert bool((ids[::3] == 1).all()) and int(ids.sum(dtype=torch.int64)) == ones and int(ids.min()) == 0
    assert float(w.min()) == 1.0 and float(w.max()) == 1.0
    grad = torch.full_like(logits, float("nan"))
    ctx.route_grad(B.make_route("sigmoid", False, 4.0), logits, ids, w, grad)     # 4 s (1 - s): 1 at a logit of 0, 0.7864 at 1
    assert ctx.device_status() == B.STRATA_OK
    want = torch.tensor(4 * 0.7310585786 * (1 - 0.7310585786), device=DEV).to(torch.bfloat16)
    assert bool((grad[::3, 1] == want).all()) and bool((grad[::3, 0] == 0).all())
    assert bool((grad[1::3, 0] == 1).all()) and bool((grad[2::3, 0] == 1).all()) and float(grad[:, 1].max()) == float(want)
    assert not bool(grad[1::3, 1].any()) and not bool(grad[2::3, 1].any())
    del ctx, logits, ids, w, grad
    torch.cuda.empty_cache()


# ---- norm --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(9001, 64), (9001, 1024), (7000, 1544)])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_grad_in_place_with_rows_fetched_ahead(rows, cols, residual):
    """More rows than the GPU holds at once, so that stages are refilled (in rows of one warp and of several): results that
    overwrite an operand are those that go elsewhere, time after time, and both are the formula's."""
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    g = base.gen(rows + cols)
    h, dy, r = (base.randn(g, rows, cols).to(torch.bfloat16) for _ in range(3))
    r = r if residual else None
    w = 1 + 0.2 * base.randn(g, cols)
    dx, dw = torch.empty_like(h), torch.empty(cols, device=DEV)
    ctx.norm_grad(dy, h, w, 1e-6, dx, dw, dresidual=r)
    want, dwant = ref.norm_grad(base.f64(dy), base.f64(h), base.f64(w), 1e-6, base.f64(r) if residual else None)
    h64, dy64 = base.f64(h), base.f64(dy)
    rstd = 1 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-6)
    hat, gg = h64 * rstd, np.abs(dy64 * base.f64(w))
    terms = rstd * (gg + np.abs(hat) * (gg * np.abs(hat)).mean(1, keepdims=True)) + (np.abs(base.f64(r)) if residual else 0)
    assert np.all(np.abs(base.f64(dx) - want) <= base.half_ulp(want) + 2.0 ** -18 * terms)
    assert np.all(np.abs(base.f64(dw) - dwant) <= (rows + 8) * U * np.abs(dy64 * hat).sum(0) + 8 * U * np.abs(dwant))
    for _ in range(8):
        for target in ("dy", "r") if residual else ("dy",):
            d2, r2, dw2 = dy.clone(), r.clone() if residual else None, torch.empty_like(dw)
            out = d2 if target == "dy" else r2
            ctx.norm_grad(d2, h, w, 1e-6, out, dw2, dresidual=r2)
            assert torch.equal(out, dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("rows", [3, 2500])
def test_norm_codes_of_a_zero_row_without_eps(kind, rows):
    """mean(h^2) + eps = 0: the reciprocal root is infinite, codes and scale of the row are zero all the same."""
    cols = 1544
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    x = base.randn(base.gen(6), rows, cols).to(torch.bfloat16)
    x[1] = 0
    weight = torch.ones(cols, device=DEV)
    for residual in (None, torch.zeros_like(x)):
        q, scale = torch.empty((rows, cols), dtype=base.CODES[kind], device=DEV), torch.full((rows,), float("nan"), device=DEV)
        ctx.norm(x, weight, 0.0, residual=residual, residual_out=None if residual is None else torch.empty_like(x), q=q, q_scale=scale)
        assert not q[1].view(torch.uint8).any() and float(scale[1]) == 0.0
        assert bool(torch.isfinite(scale).all()) and bool((scale[torch.arange(rows) != 1] > 0).all())


# Long rows in both kinds of threads: the rule's edges in columns and rows.
@pytest.mark.parametrize("rows,cols,residual,out", [
    (4096, 10240, True, "e4m3"), (4096, 10248, True, "int8"), (4096, 10248, True, "both"), (4095, 10248, True, "e4m3"),
    (4097, 16384, True, "e4m3"), (4096, 16392, True, "int8"), (2048, 8192, False, "bf16"), (2048, 8200, False, "bf16"),
    (2048, 10248, False, "bf16"), (2048, 10248, True, "bf16")])
def test_norm_of_long_rows(rows, cols, residual, out):
    base.test_norm_against_64_bits(rows, cols, residual, out)
