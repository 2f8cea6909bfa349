"""4-bit rows through the whole path, as a layer uses them: quantiser -> layout -> dispatch -> products -> quantiser -> product ->
combine, the balance loss beside it, captured and replayed, and the bounded waits of the 4-bit products.

Tolerance of the layer against fp32 weights, before the first run: e2m1 codes are half a step off at most, 1/4 of a value at 1 and
2, 1/6 at 3; over a block of normal values with its largest near 6 the error is about 11.2 % of their rms for mxfp4 and 9.5 % for
nvfp4 (root mean square over 6.4 million normal values, computed from the format).  A product's error adds the row's and the
weights': sqrt(2) times that; three products in a chain, gate and up in the same factor: four times the single error as in
test_gpu_example.py: 45 % and 38 %."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2607_26444_b200 import binding as B
from paper_2607_26444_b200 import build as strata_build

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
sys.path.insert(0, HERE)
sys.path.insert(0, os.path.join(ROOT, "examples"))
import rows4_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["mxfp4", "nvfp4"]


@pytest.mark.parametrize("kind,limit", [("mxfp4", 0.45), ("nvfp4", 0.38)])
@pytest.mark.parametrize("size", [["--tokens", "1", "--ranks", "1", "--hidden", "256", "--inner", "128"],
                                  ["--tokens", "77", "--hidden", "544", "--inner", "224", "--experts", "8", "--topk", "2"],
                                  ["--tokens", "300"]])
def test_example_layer(kind, limit, size):
    import moe_layer
    assert moe_layer.main(size + ["--kind", kind, "--steps", "2"]) < limit


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("R,T,H,E,K", [(1, 1, 32, 2, 1), (2, 30, 288, 8, 3), (4, 50, 1056, 16, 4), (2, 300, 7168, 8, 2)])
def test_dispatch_moves_rows_whole(kind, R, T, H, E, K):
    ctx = B.MoEContext(R, T, H, E, K, dispatch_dtype=B.STRATA_MXF4_ROW if kind == "mxfp4" else B.STRATA_NVF4_ROW)
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    size = B.row4_bytes(H, kind)
    sent = torch.randint(0, 256, (R, T, size), generator=g, device=DEV).to(torch.uint8)
    x = torch.randn((R, T, H), generator=g, device=DEV).to(torch.bfloat16)
    ctx.quantize_rows4(x, B.q4_rows(sent, H, kind))
    recv = torch.zeros((ctx.recv_rows, size), dtype=torch.uint8, device=DEV)
    ctx.register(recv)
    ids = torch.argsort(torch.rand((R * T, E), generator=g, device=DEV), dim=1)[:, :K].to(torch.int32).reshape(R, T, K).contiguous()
    lay = ctx.layout(ids)
    ctx.dispatch(lay, sent, recv)
    assert ctx.device_status() == B.STRATA_OK
    token = torch.arange(R * T, device=DEV).repeat_interleave(K)
    assert torch.equal(recv[lay.dst_row.flatten().long()], sent.reshape(R * T, size)[token])
    back = torch.empty((ctx.recv_rows, H), device=DEV)
    ctx.dequantize_rows4(B.q4_rows(recv, H, kind), back)
    codes, bits, rows = ref.quantize(x.reshape(R * T, H).float().cpu().numpy().astype(np.float64), kind)
    unit = ref.block_values(bits, kind) * (1.0 if rows is None else rows[:, None])
    want = ref.VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0) * np.repeat(unit, ref.BLOCK[kind], axis=1)
    got = back[lay.dst_row.flatten().long()].cpu().numpy()
    assert np.all(np.abs(got - want[token.cpu().numpy()]) <= 2.0 ** -23 * np.abs(want[token.cpu().numpy()]))


@pytest.mark.parametrize("kind", KINDS)
def test_layer_is_captured_and_replayed(kind):
    """The whole layer and its router's gradient in one graph, replayed on new hidden states, against the same calls one by one."""
    import moe_layer
    layer = moe_layer.MoELayer(2, 40, 256, 160, 8, 2, kind)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    draw = lambda: torch.randn((2, 40, 256), generator=g, device=DEV).to(torch.bfloat16)   # noqa: E731
    x, res, dgate = draw(), draw(), torch.randn((2, 40, 2), generator=g, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward(x, res)
        layer.balance(dgate)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.forward(x, res)
        dlogits = layer.balance(dgate)
    x.copy_(draw())
    res.copy_(draw())
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (out, dlogits, layer.loss, layer.stats.count, layer.ids)]
    want = [layer.forward(x, res), layer.balance(dgate), layer.loss, layer.stats.count, layer.ids]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert layer.ctx.device_status() == B.STRATA_OK
    assert int(layer.stats.count.sum()) == 2 * 40 * 2


def product(tokens, inner, seed, kind="mxfp4", E=4, K=2, channels=544):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    ctx = B.MoEContext(1, tokens, 8, E, K)
    ids = torch.argsort(torch.rand((tokens, E), generator=g, device=DEV), dim=1)[:, :K].to(torch.int32).contiguous()
    lay = ctx.layout(ids)
    a, w = B.empty_rows4((tokens * K,), inner, kind), B.empty_rows4((E, channels), inner, kind)
    x = torch.randn((tokens * K, inner), generator=g, device=DEV).to(torch.bfloat16)
    ctx.quantize_rows4(torch.randn((E, channels, inner), generator=g, device=DEV).to(torch.bfloat16), w)
    out = torch.zeros((tokens * K, channels // 2), dtype=torch.bfloat16, device=DEV)

    def call():
        ctx.quantize_rows4(x, a)
        ctx.expert_matmul4(lay, a, w, out, gated=True)
        return out
    return ctx, call, x


@pytest.mark.parametrize("tokens,inner", [(20, 1024), (500, 512), (3000, 1024), (3000, 4608)])
def test_products_are_captured_and_replayed(tokens, inner):
    """One CTA per tile and pairs of them, in a graph beside the calls one by one."""
    ctx, call, x = product(tokens, inner, 5)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    x.copy_(torch.randn(x.shape, device=DEV).to(torch.bfloat16))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    assert torch.equal(call(), got) and bool(got.any())
    assert ctx.device_status() == B.STRATA_OK


def test_products_on_two_streams_at_once():
    """Two contexts, each with its own workspace, on two streams: pairs of CTAs of both share the GPU."""
    cases = [product(3000, 2048, 1), product(2500, 4352, 2, "nvfp4")]
    want = []
    for _, call, _ in cases:
        want.append(call().clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        for stream, (_, call, _) in zip(streams, cases):
            with torch.cuda.stream(stream):
                call()
    torch.cuda.synchronize()
    for (ctx, call, _), w in zip(cases, want):
        assert ctx.device_status() == B.STRATA_OK
        assert torch.equal(call(), w)


def test_products_in_a_budget_of_sms():
    """Grids for 1, 2, 3 and 20 SMs (an odd number leaves one without a partner) give the same rows."""
    for tokens, inner in ((40, 512), (2000, 1024)):
        ctx, call, _ = product(tokens, inner, 9)
        want = call().clone()
        for n in (1, 2, 3, 20, 0):
            ctx.sm_budget(n)
            got = call()
            # another tile shape sums in another order: binary32 roundings, then one to bf16
            assert torch.allclose(got.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -9 * float(want.float().abs().max()))
        assert ctx.device_status() == B.STRATA_OK


def test_router_gradient_of_loss_and_gate_weights_together():
    """balance() = the gradient of the gate weights plus that of the losses, each against the 64-bit formulas."""
    import layer_reference
    import moe_layer
    layer = moe_layer.MoELayer(2, 30, 128, 64, 16, 4, "mxfp4")
    x, res = (torch.randn((2, 30, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    layer.forward(x, res)
    dgate = torch.randn((2, 30, 4), device=DEV)
    got = layer.balance(dgate).float().cpu().numpy().astype(np.float64)
    logits = layer.logits.float().cpu().numpy().astype(np.float64)
    ids = layer.ids.cpu().numpy()
    route = layer_reference.route_grad(logits.reshape(60, 16), ids.reshape(60, 4), dgate.cpu().numpy().reshape(60, 4), "sigmoid", True, 1.0)
    loss, count, _, _, db, dz = ref.balance(logits, ids, "sigmoid", 0.01, 0.001)
    want = route.reshape(2, 30, 16) + db + dz
    # both gradients are stored in bf16: half a step (2^-8) of each, and a few binary32 roundings of their terms
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + np.abs(route.reshape(2, 30, 16))) + 2.0 ** -16 * np.abs(route).max())
    assert np.array_equal(layer.stats.count.cpu().numpy(), count)
    np.testing.assert_allclose(layer.loss.cpu().numpy(), loss, rtol=1e-5)


@pytest.mark.parametrize("kind", ["matmul4", "matmul4_pair"])
def test_a_wait_that_runs_out_reports_timeout_and_the_context_recovers(kind):
    env = dict(os.environ, STRATA_MOE_LIB=strata_build.build_test_hooks())
    r = subprocess.run([sys.executable, os.path.join(HERE, "rows4_timeout_child.py"), kind], env=env, capture_output=True, text=True,
                       timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-3000:]
    res = json.loads([line for line in r.stdout.splitlines() if line.startswith("{")][-1])
    assert res["status_before"] == B.STRATA_OK
    assert res["status_after_injection"] == B.STRATA_ERR_TIMEOUT
    assert res["status_read_again"] == B.STRATA_OK
    assert res["header_words_after_recovery"] == [0] * 11
    assert res["same_afterwards"] and res["status_after_normal_call"] == B.STRATA_OK
