"""Refusals of the 4-bit operators and of the balance loss, through a host-only context and through the torch-level calls: every
argument error is returned before anything is launched, and valid arguments get as far as the launch."""
import types

import pytest
import torch

from paper_2607_26444_b200 import binding as B
from paper_2607_26444_b200 import build as strata_build

P = 0x7D00_0000_0000            # never dereferenced
OK, INVALID, SHAPE, ALIGN, CAP, WS, CUDA = (B.STRATA_OK, B.STRATA_ERR_INVALID_ARG, B.STRATA_ERR_SHAPE, B.STRATA_ERR_ALIGNMENT,
                                            B.STRATA_ERR_CAPACITY, B.STRATA_ERR_WORKSPACE, B.STRATA_ERR_CUDA)
MX, NV = B.STRATA_T_MXF4, B.STRATA_T_NVF4


@pytest.fixture(scope="module", autouse=True)
def built():
    strata_build.build()


def make_ctx(workspace=True, **kw):
    shape = dict(R=2, T=64, H=256, E=16, K=4, dt=B.STRATA_BF16, align=0, flags=0, cap=0)
    shape.update(kw)
    rc, h = B.strata_ctx_create(B.strata_moe_shape(*shape.values()), -1)
    assert rc == OK
    if workspace:
        assert B.strata_ctx_set_workspace(h, 0x7B00_0000_0000, 1 << 20) == OK
    return h


@pytest.fixture
def ctx():
    h = make_ctx()
    yield h
    rc, n = B.strata_ctx_launch_count(h)
    assert rc == OK and n == 0
    B.strata_ctx_destroy(h)


def rows4(type=MX, cols=256, **kw):
    q = dict(codes=P, block=P, scale=P if type == NV else None, code_stride=cols // 2,
             block_stride=-(-cols // (32 if type == MX else 16) // 16) * 16, scale_stride=1)
    q.update(kw)
    return B.strata_rows4(*q.values())


ROWS4_REFUSALS = [
    (dict(), CUDA), (dict(codes=None), INVALID), (dict(block=None), INVALID), (dict(codes=P + 8), ALIGN), (dict(block=P + 4), ALIGN),
    (dict(code_stride=112), SHAPE), (dict(code_stride=136), SHAPE), (dict(code_stride=144), CUDA), (dict(code_stride=1 << 40), SHAPE),
    (dict(block_stride=0), SHAPE), (dict(block_stride=24), SHAPE), (dict(block_stride=32), CUDA), (dict(block_stride=1 << 40), SHAPE)]


@pytest.mark.parametrize("type", [MX, NV])
@pytest.mark.parametrize("change,want", ROWS4_REFUSALS)
def test_rows4_refusals(ctx, type, change, want):
    q = rows4(type, **change)
    assert B.strata_quantize_rows4(ctx, P, 256, 10, 256, type, q, None, None) == want
    assert B.strata_dequantize_rows4(ctx, q, 10, 256, type, P, 0, 256, None, None) == want
    args = dict(type=type, gated=0, inner=256, channels=128, a_rows=512, a=rows4(type), w=q, out=P, out_stride=128)
    lay = B.strata_moe_layout_t(P, P, P, P, None, P, None)
    assert B.strata_moe_expert_matmul4(ctx, lay, B.strata_matmul4_args(*args.values()), None) == want
    args.update(a=q, w=rows4(type))
    assert B.strata_moe_expert_matmul4(ctx, lay, B.strata_matmul4_args(*args.values()), None) == want


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(x=None), INVALID), (dict(rows=0, x=None), OK), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE),
    (dict(cols=248, xs=256), SHAPE), (dict(cols=32800, xs=32800), SHAPE), (dict(xs=248), SHAPE), (dict(xs=260), SHAPE),
    (dict(type=2), INVALID), (dict(type=6), INVALID), (dict(x=P + 8), ALIGN), (dict(n=P + 2), ALIGN), (dict(n=P + 4), CUDA)])
def test_quantize_refusals(ctx, change, want):
    kw = dict(x=P, xs=256, rows=10, cols=256, type=NV, n=None)
    kw.update(change)
    assert B.strata_quantize_rows4(ctx, kw["x"], kw["xs"], kw["rows"], kw["cols"], kw["type"], rows4(NV), kw["n"], None) == want
    assert B.strata_quantize_rows4(None, P, 256, 10, 256, NV, rows4(NV), None, None) == INVALID


def test_quantize_scales_of_rows(ctx):
    """mxfp4 has none, nvfp4 needs them; read, either may have them."""
    call = lambda q, t: B.strata_quantize_rows4(ctx, P, 256, 10, 256, t, q, None, None)   # noqa: E731
    assert call(rows4(MX, scale=P), MX) == INVALID and call(rows4(NV, scale=None), NV) == INVALID
    assert call(rows4(NV, scale=P + 2), NV) == ALIGN and call(rows4(NV, scale_stride=0), NV) == SHAPE
    for q, t in ((rows4(MX, scale=P), MX), (rows4(NV, scale=None), NV)):
        assert B.strata_dequantize_rows4(ctx, q, 10, 256, t, P, 1, 256, None, None) == CUDA


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(out=None), INVALID), (dict(t=2), INVALID), (dict(t=1, s=260), CUDA), (dict(s=260), SHAPE), (dict(s=248), SHAPE),
    (dict(out=P + 8), ALIGN), (dict(rows=0, out=None), OK), (dict(rows=-1), SHAPE), (dict(n=P + 1), ALIGN)])
def test_dequantize_refusals(ctx, change, want):
    kw = dict(rows=10, out=P, t=0, s=256, n=None)
    kw.update(change)
    assert B.strata_dequantize_rows4(ctx, rows4(), kw["rows"], 256, MX, kw["out"], kw["t"], kw["s"], kw["n"], None) == want


@pytest.mark.parametrize("change,want", [
    (dict(), CUDA), (dict(type=3), INVALID), (dict(gated=2), INVALID), (dict(out=None), INVALID), (dict(out=P + 1), ALIGN),
    (dict(inner=240), SHAPE), (dict(inner=0), SHAPE), (dict(inner=131104), SHAPE), (dict(channels=0), SHAPE),
    (dict(channels=127, gated=1), SHAPE), (dict(channels=(1 << 24) + 2), SHAPE), (dict(out_stride=127), SHAPE),
    (dict(gated=1, out_stride=64), CUDA), (dict(a_rows=511), CAP), (dict(a_rows=1 << 31), SHAPE),
    (dict(w=rows4(code_stride=1 << 36)), SHAPE), (dict(w=rows4(block_stride=1 << 36)), SHAPE),
    (dict(w=rows4(code_stride=1 << 39), channels=1 << 24, out_stride=1 << 24), SHAPE),             # their product is 2^63
    (dict(w=rows4(block_stride=(1 << 40) - 16), channels=1 << 24, out_stride=1 << 24), SHAPE)])
def test_matmul_refusals(ctx, change, want):
    kw = dict(type=MX, gated=0, inner=256, channels=128, a_rows=512, a=rows4(), w=rows4(), out=P, out_stride=128)
    kw.update(change)
    lay = B.strata_moe_layout_t(P, P, P, P, None, P, None)
    assert B.strata_moe_expert_matmul4(ctx, lay, B.strata_matmul4_args(*kw.values()), None) == want


def test_matmul_needs_layout_and_workspace():
    args = B.strata_matmul4_args(MX, 0, 256, 128, 512, rows4(), rows4(), P, 128)
    h = make_ctx(workspace=False)
    assert B.strata_moe_expert_matmul4(h, B.strata_moe_layout_t(None, P, P, P, None, P, None), args, None) == INVALID
    assert B.strata_moe_expert_matmul4(h, B.strata_moe_layout_t(P, None, P, P, None, P, None), args, None) == INVALID
    assert B.strata_moe_expert_matmul4(h, B.strata_moe_layout_t(P, P, P, P, None, P, None), args, None) == WS
    B.strata_ctx_destroy(h)


BALANCE = dict(score=0, per_rank=1, weight=0.1, z=0.1, logits=P, type=1, stride=16, ids=P, loss=P, count=P, tokens=P, prob=P,
               scratch=P, nbytes=1 << 30, dloss=P, add=P, add_stride=16, dlogits=P, dstride=16)


@pytest.mark.parametrize("change,loss,grad", [
    (dict(), CUDA, CUDA), (dict(score=2), INVALID, INVALID), (dict(per_rank=2), INVALID, INVALID),
    (dict(weight=float("nan")), INVALID, INVALID), (dict(z=float("inf")), INVALID, INVALID), (dict(logits=None), INVALID, INVALID),
    (dict(ids=None), INVALID, INVALID), (dict(count=None), INVALID, INVALID), (dict(tokens=None), INVALID, INVALID),
    (dict(prob=None), INVALID, CUDA), (dict(loss=None), INVALID, CUDA), (dict(scratch=None), INVALID, CUDA),
    (dict(nbytes=16), CAP, CUDA), (dict(type=2), INVALID, INVALID), (dict(stride=15), SHAPE, SHAPE), (dict(logits=P + 2), ALIGN, ALIGN),
    (dict(ids=P + 2), ALIGN, ALIGN), (dict(scratch=P + 8), ALIGN, CUDA), (dict(dlogits=None), CUDA, INVALID),
    (dict(dstride=15), CUDA, SHAPE), (dict(add_stride=15), CUDA, SHAPE), (dict(add=None, add_stride=0), CUDA, CUDA),
    (dict(dloss=None), CUDA, CUDA), (dict(dloss=P + 2), CUDA, ALIGN), (dict(add=P + 1, type=0), CUDA, ALIGN)])
def test_balance_refusals(ctx, change, loss, grad):
    k = {**BALANCE, **change}
    params = B.strata_balance_params(k["score"], k["per_rank"], k["weight"], k["z"])
    stats = B.strata_balance_stats(k["count"], k["tokens"], k["prob"])
    assert B.strata_moe_balance_loss(ctx, params, k["logits"], k["type"], k["stride"], k["ids"], k["loss"], stats, k["scratch"],
                                     k["nbytes"], None) == loss
    assert B.strata_moe_balance_grad(ctx, params, k["logits"], k["type"], k["stride"], k["ids"], stats, k["dloss"], k["add"],
                                     k["add_stride"], k["dlogits"], k["dstride"], None) == grad


def test_balance_scratch_and_parameters(ctx):
    rc, n = B.strata_moe_balance_scratch_bytes(ctx, B.make_balance())
    assert rc == OK and n > 0
    assert B.strata_moe_balance_scratch_bytes(ctx, B.make_balance(weight=float("nan")))[0] == INVALID
    with pytest.raises(ValueError):
        B.make_balance("relu")


@pytest.mark.parametrize("kind,dt", [("mxfp4", B.STRATA_MXF4_ROW), ("nvfp4", B.STRATA_NVF4_ROW)])
def test_rows_that_dispatch_moves(kind, dt):
    """Shapes, the size of a row (what a rank's view of the receive buffer is cut by), and the views of its parts."""
    import numpy as np
    assert B.strata_ctx_create(B.strata_moe_shape(2, 64, 272, 16, 4, dt), -1)[0] == SHAPE       # H % 32
    assert B.strata_ctx_create(B.strata_moe_shape(2, 64, 256, 16, 4, 5), -1)[0] == SHAPE        # no such type
    for H in (32, 288, 7168):
        h = make_ctx(H=H, dt=dt)
        rc, base, rows = B.strata_moe_recv_view(h, np.array([0, 3, 10], np.int32), 1, P)
        size = B.row4_bytes(H, kind)
        assert rc == OK and rows == 7 and base == P + 3 * size and size % 32 == 0
        assert B.strata_moe_dispatch(h, B.strata_moe_layout_t(P, P, P, P, None, P, None), P, P, None, 512, None) == B.STRATA_ERR_NOT_REGISTERED
        B.strata_ctx_destroy(h)
        q = B.q4_rows(torch.zeros((3, 4, size), dtype=torch.uint8), H, kind)
        assert q.rows == 12 and q.cols == H and q.c.code_stride == q.c.block_stride == size
        if kind == "nvfp4":
            assert q.c.scale_stride == size // 4 and q.c.scale - q.c.codes >= H // 2 + H // 16 and (q.c.scale - q.c.codes) % 16 == 0
            assert q.c.scale - q.c.codes + 4 <= size
    with pytest.raises(ValueError):
        B.q4_rows(torch.zeros((3, 100), dtype=torch.uint8), 128, kind)


def test_rows4_are_checked_before_any_address_is_taken():
    codes, block = torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 16), dtype=torch.uint8)
    mx, nv = block.view(torch.float8_e8m0fnu), block.view(torch.float8_e4m3fn)
    assert B.Rows4(codes, mx[:, :4]).type == MX and B.Rows4(codes, nv[:, :8]).type == NV
    assert B.Rows4(codes.view(torch.float4_e2m1fn_x2), mx[:, :4]).cols == 128
    for args in ((codes.to(torch.int8), mx[:, :4]), (codes, block[:, :4]), (codes, mx[:, :8]), (codes, nv[:, :4]), (codes, mx[:3, :4]),
                 (codes[:, :8], mx[:, :1]), (codes, mx[:, :4], torch.ones(4, dtype=torch.bfloat16)), (codes, mx[:, :4], torch.ones(3)),
                 (codes, mx[:, :4], torch.ones(1).expand(4)), (codes.t(), mx[:, :4])):
        with pytest.raises(ValueError):
            B.Rows4(*args)
    for bad in ("e2m1", "int8"):
        with pytest.raises(ValueError):
            B.empty_rows4((4,), 64, bad, device="cpu")
        with pytest.raises(ValueError):
            B.row4_bytes(64, bad)


def host_context():
    def reached(*args):
        raise AssertionError("the call reached the library")
    names = ("quantize_rows4", "dequantize_rows4", "moe_expert_matmul4", "moe_balance_loss", "moe_balance_grad")
    return types.SimpleNamespace(h=None, _c=types.SimpleNamespace(**{"strata_" + n: reached for n in names}), _stream=lambda: 0,
                                 n_tok=8, n_items=16, E=16, K=2, R=2, _balance_stats=lambda p, s: B.MoEContext._balance_stats(
                                     types.SimpleNamespace(R=2, E=16), p, s))


def test_torch_level_refusals():
    c, M = host_context(), B.MoEContext
    q = B.empty_rows4((8,), 64, "mxfp4", device="cpu")
    x = torch.zeros((8, 64), dtype=torch.bfloat16)
    for bad in (x[:7], x[:, :32], x.float()):
        with pytest.raises(ValueError):
            M.quantize_rows4(c, bad, q)
    for bad in (x[:7], x[:, :32], x.half()):
        with pytest.raises(ValueError):
            M.dequantize_rows4(c, q, bad)
    w = B.empty_rows4((16, 10), 64, "mxfp4", device="cpu")
    lay = types.SimpleNamespace(c=B.strata_moe_layout_t())
    out = torch.zeros((8, 10), dtype=torch.bfloat16)
    for a, b, o, gated in ((q, B.empty_rows4((16, 10), 64, "nvfp4", device="cpu"), out, False), (q, q, out, False),
                           (q, B.empty_rows4((16, 10), 96, "mxfp4", device="cpu"), out, False), (q, w, out[:7], False),
                           (q, B.empty_rows4((15, 10), 64, "mxfp4", device="cpu"), out, False), (q, w, out, True), (q, w, out.float(), False)):
        with pytest.raises(ValueError):
            M.expert_matmul4(c, lay, a, b, o, gated=gated)
    with pytest.raises(AssertionError):
        M.expert_matmul4(c, lay, q, w, out)
    params, other = B.make_balance(per_rank=True), B.make_balance()
    stats = B.BalanceStats(2, 16, 64, "cpu")
    logits, ids, loss = torch.zeros((8, 16)), torch.zeros((8, 2), dtype=torch.int32), torch.zeros(2)
    for p, l, i, o, s in ((other, logits, ids, loss, stats), (params, logits[:7], ids, loss, stats), (params, logits.half(), ids, loss, stats),
                          (params, logits, ids.long(), loss, stats), (params, logits, ids[:7], loss, stats),
                          (params, logits, ids, loss[:1], stats), (params, logits, ids, loss.double(), stats)):
        with pytest.raises(ValueError):
            M.balance_loss(c, p, l, i, o, s)
    for kw in (dict(dlogits=logits.to(torch.bfloat16)), dict(dlogits=logits, add=logits.to(torch.bfloat16)), dict(dlogits=logits[:4]),
               dict(dlogits=logits, dloss=torch.zeros(1)), dict(dlogits=logits, add=logits[:, :8])):
        with pytest.raises(ValueError):
            M.balance_grad(c, params, logits, ids, stats, **kw)
    with pytest.raises(AssertionError):
        M.balance_grad(c, params, logits, ids, stats, logits)
