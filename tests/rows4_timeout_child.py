"""Child process of tests/test_gpu_layer4.py: runs with STRATA_MOE_LIB pointing at the test-hooks build (see layer_timeout_child.py).

The first load of one launch is expected to bring 16 bytes more than it does, so that the waits of the 4-bit products run out: alone in
a CTA (few rows per expert) and in a pair of CTAs (many).  Prints one JSON line."""
import ctypes
import json
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_26444_b200 import binding as B  # noqa: E402

DEV = "cuda:0"


def matmul_call(tokens):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    E, K, inner, channels = 4, 2, 2048, 512
    ctx = B.MoEContext(1, tokens, 8, E, K)
    ids = torch.argsort(torch.rand((tokens, E), generator=g, device=DEV), dim=1)[:, :K].to(torch.int32).reshape(1, tokens, K).contiguous()
    lay = ctx.layout(ids)
    a, w = B.empty_rows4((tokens * K,), inner, "mxfp4"), B.empty_rows4((E, channels), inner, "mxfp4")
    ctx.quantize_rows4(torch.randn((tokens * K, inner), generator=g, device=DEV).to(torch.bfloat16), a)
    ctx.quantize_rows4(torch.randn((E, channels, inner), generator=g, device=DEV).to(torch.bfloat16), w)

    def call():
        out = torch.zeros((tokens * K, channels), dtype=torch.bfloat16, device=DEV)
        ctx.expert_matmul4(lay, a, w, out)
        return out
    return ctx, call


def main(kind):
    hook = B.lib().strata_test_inject_short_load4
    hook.argtypes, hook.restype = [ctypes.c_int], None
    ctx, call = matmul_call(20 if kind == "matmul4" else 6000)
    before = call()
    res = {"kind": kind, "status_before": ctx.device_status()}
    hook(1)
    call()
    res["status_after_injection"] = ctx.device_status()
    res["status_read_again"] = ctx.device_status()
    res["header_words_after_recovery"] = ctx.workspace[:44].view(torch.int32).cpu().tolist()
    res["same_afterwards"] = bool(torch.equal(call(), before))
    res["status_after_normal_call"] = ctx.device_status()
    print(json.dumps(res), flush=True)


if __name__ == "__main__":
    main(sys.argv[1])
