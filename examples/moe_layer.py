"""One feed-forward layer of a mixture of experts on one GPU, forward pass, experts in 8 or in 4 bits:

    residual addition + RMS norm -> router -> routing layout -> dispatch -> gate and up products -> silu(gate) * up
    -> rows to 8 (4) bits -> down product -> gate-weighted combine

In 8 bits the hidden states leave the norm twice: in bf16 for the router, and as 8-bit rows that carry their scale, which
dispatch moves (half the bytes of bf16).  In 4 bits (mxfp4, nvfp4) the quantiser makes the rows that dispatch moves, a
quarter of the bytes, with their block scales.  The receive buffer is what the experts' products read; nothing is copied
in between, and no step waits for the host.

balance() adds what training asks of the router: the balance loss of the batch, the counts per expert, and the gradient of
the logits from the loss and from the gate weights together.

    python examples/moe_layer.py [--tokens 128] [--hidden 1024] [--inner 512] [--experts 32] [--topk 4]
                                 [--kind int8|e4m3|mxfp4|nvfp4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_26444_b200 import binding as B  # noqa: E402

CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
ROWS4 = {"mxfp4": B.STRATA_MXF4_ROW, "nvfp4": B.STRATA_NVF4_ROW}


def to_codes(weight, kind):
    """8-bit weights [E, channels, inner] and a scale per output channel, made once when the weights are loaded."""
    limit = 127.0 if kind == "int8" else 448.0
    scale = weight.abs().amax(dim=-1).clamp_min(1e-12) / limit
    units = weight / scale[..., None]
    return (units.round().to(torch.int8) if kind == "int8" else units.to(torch.float8_e4m3fn)), scale.contiguous()


class MoELayer:
    """Weights and buffers of one layer for batches of R ranks x T tokens."""

    def __init__(self, R, T, hidden, inner, experts, topk, kind="int8", device="cuda:0", seed=0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, generator=g, device=device)
        self.kind, self.four = kind, kind in ROWS4
        self.ctx = B.MoEContext(R, T, hidden, experts, topk, dispatch_dtype=ROWS4.get(kind, B.STRATA_Q8_ROW),
                                allow_unrouted=True)
        self.norm_weight = 1.0 + 0.1 * normal(hidden)
        self.router = (normal(experts, hidden) / hidden ** 0.5).to(torch.bfloat16)
        self.bias = 0.01 * normal(experts)
        self.gate_up = normal(experts, 2 * inner, hidden) / hidden ** 0.5
        self.down = normal(experts, hidden, inner) / inner ** 0.5
        if self.four:
            self.w1, self.w2 = self.to_rows4(self.gate_up), self.to_rows4(self.down)
        else:
            self.w1, self.s1 = to_codes(self.gate_up, kind)
            self.w2, self.s2 = to_codes(self.down, kind)
        self.params = B.make_route("sigmoid", renormalise=True, scale=1.0, n_group=4, topk_group=2, group_score="top2")
        rows, bf = self.ctx.recv_rows, dict(dtype=torch.bfloat16, device=device)
        self.h, self.y, self.out = (torch.empty((R, T, hidden), **bf) for _ in range(3))
        row_bytes = B.row4_bytes(hidden, kind) if self.four else hidden + B.STRATA_Q8_TRAILER
        self.sent = torch.zeros((R, T, row_bytes), dtype=torch.uint8, device=device)
        self.recv = torch.zeros((rows, row_bytes), dtype=torch.uint8, device=device)
        self.ctx.register(self.recv)
        self.ids = torch.empty((R, T, topk), dtype=torch.int32, device=device)
        self.gate = torch.empty((R, T, topk), dtype=torch.float32, device=device)
        self.mid = torch.empty((rows, inner), **bf)
        if self.four:
            self.sent4, self.recv4 = B.q4_rows(self.sent, hidden, kind), B.q4_rows(self.recv, hidden, kind)
            self.mid4 = B.empty_rows4((rows,), inner, kind, device)
        else:
            self.mid_q = torch.empty((rows, inner), dtype=CODES[kind], device=device)
            self.mid_scale = torch.empty(rows, dtype=torch.float32, device=device)
        self.back = torch.empty((rows, hidden), **bf)
        self.lay = self.ctx.new_layout()
        self.balance_params = B.make_balance("sigmoid", weight=0.01, z_weight=0.001, per_rank=True)
        self.stats = self.ctx.balance_stats(self.balance_params)
        self.loss = torch.empty(2, dtype=torch.float32, device=device)

    def to_rows4(self, weight):
        """4-bit weights [E, channels, inner], made once when the weights are loaded."""
        q = B.empty_rows4(weight.shape[:-1], weight.shape[-1], self.kind, weight.device)
        self.ctx.quantize_rows4(weight.to(torch.bfloat16), q)
        return q

    def forward(self, x, residual):
        """x, residual: bf16 [R, T, hidden].  Returns the experts' combined output; the new residual is self.h."""
        ctx = self.ctx
        q, q_scale = (None, None) if self.four else B.q8_rows(self.sent, CODES[self.kind])
        ctx.norm(x, self.norm_weight, 1e-6, out=self.y, residual=residual, residual_out=self.h, q=q, q_scale=q_scale)
        if self.four:
            ctx.quantize_rows4(self.y, self.sent4)
        self.logits = torch.matmul(self.y, self.router.t())
        ctx.route(self.params, self.logits, self.ids, self.gate, bias=self.bias)
        ctx.layout(self.ids, self.lay)
        ctx.dispatch(self.lay, self.sent, self.recv)
        if self.four:
            ctx.expert_matmul4(self.lay, self.recv4, self.w1, self.mid, gated=True)
            ctx.quantize_rows4(self.mid, self.mid4, layout=self.lay)
            ctx.expert_matmul4(self.lay, self.mid4, self.w2, self.back)
        else:
            a, a_scale = B.q8_rows(self.recv, CODES[self.kind])
            ctx.expert_matmul(self.lay, a, a_scale, self.w1, self.s1, self.mid, gated=True)
            ctx.quantize_rows(self.mid, self.mid_q, self.mid_scale, layout=self.lay)
            ctx.expert_matmul(self.lay, self.mid_q, self.mid_scale, self.w2, self.s2, self.back)
        ctx.combine(self.lay, self.back, self.gate, self.out)
        return self.out

    def balance(self, dgate):
        """After forward: the losses (self.loss), the counts (self.stats.count) and the gradient of the logits, from the
        losses and from the gradient of the gate weights together."""
        dlogits = torch.empty_like(self.logits)
        self.ctx.route_grad(self.params, self.logits, self.ids, dgate, dlogits)
        self.ctx.balance_loss(self.balance_params, self.logits, self.ids, self.loss, self.stats)
        self.ctx.balance_grad(self.balance_params, self.logits, self.ids, self.stats, dlogits, add=dlogits)
        return dlogits

    def reference(self, x, residual):
        """The same layer in fp32 from the unquantised weights, with the ids that the router chose."""
        h = (x.float() + residual.float()).to(torch.bfloat16).float()
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6) * self.norm_weight
        y = y.reshape(-1, y.shape[-1])
        out = torch.zeros_like(y)
        ids, gate = self.ids.reshape(y.shape[0], -1).long(), self.gate.reshape(y.shape[0], -1)
        for e in range(self.router.shape[0]):
            tok, slot = torch.nonzero(ids == e, as_tuple=True)
            if tok.numel():
                g, u = (y[tok] @ self.gate_up[e].t()).chunk(2, dim=-1)
                out.index_add_(0, tok, (torch.nn.functional.silu(g) * u) @ self.down[e].t() * gate[tok, slot][:, None])
        return out.reshape(x.shape)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("ranks", 2), ("tokens", 128), ("hidden", 1024), ("inner", 512), ("experts", 32), ("topk", 4), ("steps", 20)):
        ap.add_argument(f"--{name}", type=int, default=default)
    ap.add_argument("--kind", choices=[*CODES, *ROWS4], default="int8")
    a = ap.parse_args(argv)
    layer = MoELayer(a.ranks, a.tokens, a.hidden, a.inner, a.experts, a.topk, a.kind)
    x, residual = (torch.randn((a.ranks, a.tokens, a.hidden), device="cuda:0").to(torch.bfloat16) for _ in range(2))
    out = layer.forward(x, residual)
    status = layer.ctx.device_status()
    if status != B.STRATA_OK:
        raise B.StrataError(status, "moe_layer")
    want = layer.reference(x, residual)
    error = float((out.float() - want).norm() / want.norm())
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(a.steps):
        layer.forward(x, residual)
    end.record()
    torch.cuda.synchronize()
    print(f"{a.ranks} x {a.tokens} tokens, hidden {a.hidden}, inner {a.inner}, {a.experts} experts, top-{a.topk}, {a.kind}: "
          f"relative error {error:.4f} against fp32 weights, {start.elapsed_time(end) / a.steps * 1e3:.1f} us per pass")
    return error


if __name__ == "__main__":
    main()
