"""Child process of tests/test_gpu_layer_timeout.py: runs with STRATA_MOE_LIB pointing at the test-hooks build.

Makes one bounded wait run out in each kernel that waits for copies (the hook makes block 0 expect 16 bytes more than its first
copy delivers; nothing faults, traps or spins without a limit) and checks that the kernel returns, that the status says
so, and that the next call on the same context gives what it gave before.  Prints one JSON line."""
import ctypes
import json
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_26444_b200 import binding as B  # noqa: E402

DEV = "cuda:0"


def matmul_call():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    E, T, K, inner, channels = 4, 96, 2, 256, 256
    ctx = B.MoEContext(1, T, 8, E, K)
    ids = torch.argsort(torch.rand((T, E), generator=g, device=DEV), dim=1)[:, :K].to(torch.int32).reshape(1, T, K).contiguous()
    lay = ctx.layout(ids)
    a = torch.randint(-100, 100, (T * K, inner), generator=g, device=DEV).to(torch.int8)
    w = torch.randint(-100, 100, (E, channels, inner), generator=g, device=DEV).to(torch.int8)
    a_s, w_s = torch.rand(T * K, generator=g, device=DEV), torch.rand((E, channels), generator=g, device=DEV)

    def call():
        out = torch.zeros((T * K, channels), dtype=torch.bfloat16, device=DEV)
        ctx.expert_matmul(lay, a, a_s, w, w_s, out)
        return out
    return ctx, call


def norm_grad_call(cols):
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    ctx = B.MoEContext(1, 1, 8, 1, 1)
    n = 7000
    x, r = (torch.randn((n, cols), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    w = torch.ones(cols, device=DEV)

    def call():
        dx, dw = torch.zeros_like(x), torch.zeros(cols, device=DEV)
        ctx.norm_grad(x, r, w, 1e-6, dx, dw, dresidual=r)
        return torch.cat([dx.float().sum(0), dw])
    return ctx, call


def main(kind):
    L = B.lib()
    hook = L.strata_test_inject_short_load if kind == "matmul" else L.strata_test_inject_short_row
    hook.argtypes, hook.restype = [ctypes.c_int], None
    ctx, call = matmul_call() if kind == "matmul" else norm_grad_call(512 if kind.endswith("warp") else 1544)
    before = call()
    res = {"kind": kind, "status_before": ctx.device_status()}
    hook(1)
    call()
    res["status_after_injection"] = ctx.device_status()
    res["status_read_again"] = ctx.device_status()
    res["header_words_after_recovery"] = ctx.workspace[:40].view(torch.int32).cpu().tolist()
    res["same_afterwards"] = bool(torch.equal(call(), before))
    res["status_after_normal_call"] = ctx.device_status()
    print(json.dumps(res), flush=True)


if __name__ == "__main__":
    main(sys.argv[1])
