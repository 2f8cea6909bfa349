"""Refusals of the layer operators (include/strata_layer.h), through a host-only context: every argument error is
returned before anything is launched, and valid arguments get as far as the launch."""
import pytest

from paper_2607_26444_b200 import binding as B
from paper_2607_26444_b200 import build as strata_build

P = 0x7D00_0000_0000            # never dereferenced
INVALID, SHAPE, ALIGN, CAP, WS, CUDA = (B.STRATA_ERR_INVALID_ARG, B.STRATA_ERR_SHAPE, B.STRATA_ERR_ALIGNMENT,
                                        B.STRATA_ERR_CAPACITY, B.STRATA_ERR_WORKSPACE, B.STRATA_ERR_CUDA)


@pytest.fixture(scope="module", autouse=True)
def built():
    strata_build.build()


def make_ctx(workspace=True, **kw):
    shape = dict(R=2, T=64, H=256, E=16, K=4, dt=B.STRATA_BF16, align=0, flags=0, cap=0)
    shape.update(kw)
    rc, h = B.strata_ctx_create(B.strata_moe_shape(*shape.values()), -1)
    assert rc == B.STRATA_OK
    if workspace:
        assert B.strata_ctx_set_workspace(h, 0x7B00_0000_0000, 1 << 20) == B.STRATA_OK
    return h


@pytest.fixture
def ctx():
    h = make_ctx()
    yield h
    rc, n = B.strata_ctx_launch_count(h)
    assert rc == B.STRATA_OK and n == 0
    B.strata_ctx_destroy(h)


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(score=2), INVALID), (dict(group_score=2), INVALID), (dict(renormalise=2), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(n_group=0), SHAPE), (dict(n_group=3), SHAPE), (dict(n_group=64), SHAPE), (dict(topk_group=0), SHAPE),
    (dict(n_group=4, topk_group=5), SHAPE), (dict(n_group=8, topk_group=1), SHAPE),      # 2 experts for 4 slots
    (dict(n_group=8, topk_group=2), CUDA),
    (dict(logits=None), INVALID), (dict(ids=None), INVALID), (dict(w=None), INVALID), (dict(type=2), INVALID),
    (dict(stride=15), SHAPE), (dict(logits=P + 2), ALIGN), (dict(logits=P + 2, type=0), CUDA), (dict(bias=P + 1), ALIGN),
    (dict(ids=P + 2), ALIGN)])
def test_route_refusals(ctx, change, want):
    kw = dict(score=0, renormalise=1, n_group=1, topk_group=1, group_score=0, scale=1.0, logits=P, type=1, stride=16,
              bias=None, ids=P, w=P)
    kw.update(change)
    params = B.strata_route_params(kw["score"], kw["renormalise"], kw["n_group"], kw["topk_group"], kw["group_score"],
                                   kw["scale"])
    assert B.strata_moe_route(ctx, params, kw["logits"], kw["type"], kw["stride"], kw["bias"], kw["ids"], kw["w"], None) == want
    if kw["bias"] is None:
        assert B.strata_moe_route_grad(ctx, params, kw["logits"], kw["type"], kw["stride"], kw["ids"], kw["w"], P, 16,
                                       None) == want
    assert B.strata_moe_route(None, params, P, 1, 16, None, P, P, None) == INVALID


def test_route_grad_refusals(ctx):
    params = B.make_route()
    assert B.strata_moe_route_grad(ctx, params, P, 1, 16, P, P, None, 16, None) == INVALID
    assert B.strata_moe_route_grad(ctx, params, P, 1, 16, P, P, P, 15, None) == SHAPE
    assert B.strata_moe_route_grad(ctx, params, P, 1, 16, P, P, P + 2, 16, None) == ALIGN
    h = make_ctx(workspace=False)
    assert B.strata_moe_route_grad(h, params, P, 1, 16, P, P, P, 16, None) == WS
    B.strata_ctx_destroy(h)
    with pytest.raises(ValueError):
        B.make_route("relu")


NORM = dict(rows=10, cols=256, weight_type=0, eps=1e-6, q_type=B.STRATA_T_INT8, x=P, residual=P, weight=P, residual_out=P,
            out=P, q=P, q_scale=P, x_stride=256, residual_stride=256, residual_out_stride=256, out_stride=256, q_stride=256,
            q_scale_stride=1)


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(x=None), INVALID), (dict(weight=None), INVALID), (dict(out=None, q=None), INVALID),
    (dict(out=None), CUDA), (dict(q=None, q_scale=None), CUDA), (dict(residual=None), INVALID),
    (dict(residual_out=None), INVALID), (dict(residual=None, residual_out=None), CUDA), (dict(q_scale=None), INVALID),
    (dict(weight_type=2), INVALID), (dict(q_type=0), INVALID), (dict(q_type=B.STRATA_T_E4M3), CUDA),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE),
    (dict(cols=252), SHAPE), (dict(cols=32776, x_stride=40000), SHAPE), (dict(x_stride=248), SHAPE),
    (dict(x_stride=260), SHAPE), (dict(out_stride=8), SHAPE), (dict(residual_stride=255), SHAPE),
    (dict(residual_out_stride=0), SHAPE), (dict(q_stride=252), SHAPE), (dict(q_scale_stride=0), SHAPE),
    (dict(x=P + 8), ALIGN), (dict(residual=P + 2), ALIGN), (dict(out=P + 4), ALIGN), (dict(weight=P + 8), ALIGN),
    (dict(q=P + 4), ALIGN), (dict(q=P + 8), CUDA), (dict(q_scale=P + 2), ALIGN),
    (dict(rows=0, x=None, out=None, q=None), B.STRATA_OK)])
def test_norm_refusals(ctx, change, want):
    kw = {**NORM, **change}
    assert B.strata_norm(ctx, B.strata_norm_args(**kw), None) == want
    assert B.strata_norm(None, B.strata_norm_args(**kw), None) == INVALID


GRAD = dict(rows=10, cols=256, weight_type=1, eps=1e-6, dy=P, h=P, weight=P, dresidual=P, dx=P, dweight=P, scratch=P,
            scratch_bytes=1 << 30, dy_stride=256, h_stride=256, dresidual_stride=256, dx_stride=256)


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(dy=None), INVALID), (dict(h=None), INVALID), (dict(dx=None), INVALID),
    (dict(dweight=None), INVALID), (dict(weight=None), INVALID), (dict(dresidual=None), CUDA),
    (dict(weight_type=3), INVALID), (dict(eps=float("inf")), INVALID), (dict(cols=12), SHAPE), (dict(rows=-5), SHAPE),
    (dict(dy_stride=128), SHAPE), (dict(h_stride=257), SHAPE), (dict(dx_stride=0), SHAPE),
    (dict(dresidual_stride=12), SHAPE), (dict(dy=P + 2), ALIGN), (dict(scratch=P + 8), ALIGN), (dict(dweight=P + 2), ALIGN)])
def test_norm_grad_refusals(ctx, change, want):
    kw = {**GRAD, **change}
    assert B.strata_norm_grad(ctx, B.strata_norm_grad_args(**kw), None) == want


def test_norm_grad_scratch(ctx):
    rc, n = B.strata_norm_grad_scratch_bytes(ctx, -1, 256)
    assert rc == SHAPE
    rc, n = B.strata_norm_grad_scratch_bytes(ctx, 0, 256)
    assert rc == B.STRATA_OK and n == 0


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID), (dict(rows=0, x=None), B.STRATA_OK),
    (dict(rows=-2), SHAPE), (dict(cols=100), SHAPE), (dict(xs=100), SHAPE), (dict(qs=100), SHAPE), (dict(t=1), INVALID),
    (dict(x=P + 8), ALIGN), (dict(q=P + 1), ALIGN), (dict(n=P + 2), ALIGN), (dict(n=P + 4), CUDA)])
def test_quantize_refusals(ctx, change, want):
    kw = dict(x=P, xs=104, rows=7, cols=104, t=B.STRATA_T_E4M3, q=P, qs=104, s=P, ss=1, n=None)
    kw.update(change)
    assert B.strata_quantize_rows(ctx, kw["x"], kw["xs"], kw["rows"], kw["cols"], kw["t"], kw["q"], kw["qs"], kw["s"],
                                  kw["ss"], kw["n"], None) == want


MATMUL = dict(type=B.STRATA_T_INT8, gated=1, inner=256, channels=128, a_rows=512, a=P, a_scale=P, w=P, w_scale=P, out=P,
              a_stride=288, a_scale_stride=72, out_stride=64)


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(type=B.STRATA_T_E4M3), CUDA), (dict(type=0), INVALID), (dict(gated=2), INVALID),
    (dict(a=None), INVALID), (dict(w=None), INVALID), (dict(a_scale=None), INVALID), (dict(w_scale=None), INVALID),
    (dict(out=None), INVALID), (dict(inner=0), SHAPE), (dict(inner=250), SHAPE), (dict(inner=131072, a_stride=131072), SHAPE),
    (dict(channels=126), CUDA), (dict(channels=126, gated=0, out_stride=126), CUDA), (dict(channels=0), SHAPE),
    (dict(channels=127, gated=0, out_stride=127), CUDA), (dict(channels=127), SHAPE), (dict(a_stride=240), SHAPE), (dict(a_stride=264), SHAPE),
    (dict(a_scale_stride=0), SHAPE), (dict(out_stride=62), SHAPE), (dict(out_stride=65), CUDA), (dict(gated=0), SHAPE),
    (dict(a_rows=511), CAP), (dict(a=P + 8), ALIGN), (dict(w=P + 8), ALIGN), (dict(out=P + 2), CUDA), (dict(out=P + 1), ALIGN),
    (dict(a_scale=P + 2), ALIGN)])
def test_matmul_refusals(ctx, change, want):
    lay = B.strata_moe_layout_t(P, P, P, P, None, P, None)
    kw = {**MATMUL, **change}
    assert B.strata_moe_expert_matmul(ctx, lay, B.strata_matmul_args(**kw), None) == want
    bad = B.strata_moe_layout_t(P, None, P, P, None, P, None)
    assert B.strata_moe_expert_matmul(ctx, bad, B.strata_matmul_args(**kw), None) == INVALID


def test_operators_need_a_workspace():
    h = make_ctx(workspace=False)
    assert B.strata_norm(h, B.strata_norm_args(**NORM), None) == CUDA             # needs none
    assert B.strata_norm_grad(h, B.strata_norm_grad_args(**GRAD), None) == WS
    lay = B.strata_moe_layout_t(P, P, P, P, None, P, None)
    assert B.strata_moe_expert_matmul(h, lay, B.strata_matmul_args(**MATMUL), None) == WS
    B.strata_ctx_destroy(h)


def test_q8_row_contexts():
    """8-bit rows with their scale behind the codes: H a multiple of 16, H + 32 bytes per row, no separate scales."""
    rc, _ = B.strata_ctx_create(B.strata_moe_shape(2, 64, 264, 16, 4, B.STRATA_Q8_ROW), -1)
    assert rc == SHAPE
    h = make_ctx(H=272, dt=B.STRATA_Q8_ROW)
    lay = B.strata_moe_layout_t(P, P, P, P, None, P, None)
    recv, rows = 0x7C00_0000_0000, 512
    assert B.strata_moe_dispatch(h, lay, P, recv, P, rows, None) == INVALID               # scales travel inside the rows
    rc, rid = B.strata_pool_register(h, recv, rows * 304 - 16)
    assert B.strata_moe_dispatch(h, lay, P, recv, None, rows, None) == B.STRATA_ERR_NOT_REGISTERED
    B.strata_pool_unregister(h, rid)
    B.strata_pool_register(h, recv, rows * 304)
    assert B.strata_moe_dispatch(h, lay, P, recv, None, rows, None) == CUDA
    import numpy as np
    rc, base, n = B.strata_moe_recv_view(h, np.array([0, 100, 512], np.int32), 1, recv)
    assert rc == B.STRATA_OK and base == recv + 100 * 304 and n == 412
    B.strata_ctx_destroy(h)


def test_binding_checks_tensors():
    import torch
    t = torch.empty((4, 6, 16), dtype=torch.bfloat16)
    assert B._strides(t) == (24, 16, 16)
    assert B._strides(t[:, :, :8]) == (24, 8, 16)
    assert B._strides(t[:, 2]) == (4, 16, 96)
    assert B._strides(t[1, 2]) == (1, 16, 16)
    for bad in (t[:, ::2, :][:, :2], t.transpose(1, 2)):
        with pytest.raises(ValueError):
            B._strides(bad)
    buf = torch.zeros((3, 48 + B.STRATA_Q8_TRAILER), dtype=torch.uint8)
    codes, scale = B.q8_rows(buf, torch.int8)
    scale[1] = 1.5
    codes[1, 47] = 3
    assert buf[1, 48:52].view(torch.float32).item() == 1.5 and buf[1, 47] == 3 and codes.shape == (3, 48)
    assert B._scale_stride(scale, 3) == 20
    with pytest.raises(ValueError):
        B._scale_stride(scale, 4)
    with pytest.raises(ValueError):
        B._code_type(buf)
    with pytest.raises(ValueError):
        B._float_type(buf)
