"""Child process of tests/test_gpu_matmul4_tiles.py: runs with STRATA_MOE_LIB pointing at the test-hooks build.

Every product runs on the tile that the command line names (-1: the one that the library chooses), against the 64-bit form and the
tolerances of test_gpu_rows4.py.  Prints one JSON line: {case: ["ok", "refused" or what went wrong, a digest of the rows]}; with a second argument "timeout"
what became of a wait that ran out."""
import ctypes
import hashlib
import json
import os
import sys

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
sys.path.insert(0, os.path.dirname(HERE))
import rows4_reference as ref  # noqa: E402
import test_gpu_rows4 as t  # noqa: E402
from paper_2607_26444_b200 import binding as B  # noqa: E402

DEV = "cuda:0"
SHAPES = {
    "least": dict(tokens=3, E=2, K=1, inner=32, channels=16),
    "odd": dict(tokens=33, E=5, K=2, inner=96, channels=132),                                   # gated: rows of out on 4 bytes
    "skewed": dict(tokens=701, E=3, K=2, inner=1056, channels=1040, skew=True),                 # a span of 32 values at the end
    "idle": dict(tokens=500, E=7, K=2, inner=288, channels=400, skew=True, allow_unrouted=True),
    "aligned": dict(tokens=130, E=6, K=2, inner=256, channels=640, R=2, segment_align=16),
    "long": dict(tokens=397, E=2, K=1, inner=4640, channels=592),                               # many stages, a partial last group of scales
    "tables": dict(tokens=600, E=512, K=1, inner=64, channels=64),                              # as many experts as the widest tile has room for
    "too_many": dict(tokens=600, E=513, K=1, inner=64, channels=64),
    "many_tiles": dict(tokens=6000, E=2, K=1, inner=64, channels=1552),                         # several tiles for every pair of CTAs
}
# rows of out: channels, their distance and the first element, for 16, 8, 4 and 2 bytes
NARROW = [(1040, 1040, 0), (1040, 1044, 0), (1044, 1044, 4), (1042, 1042, 2), (1042, 1043, 0), (1041, 1041, 1)]


def product(c, kind, gated):
    ctx, lay, a, w, out = t.matmul_case(gated=gated, kind=kind, seed=17, pad=32, **c)
    ctx.expert_matmul4(lay, a, w, out, gated=gated)
    t.check_products(lay, a, w, out, gated)
    first = out.clone()
    ctx.expert_matmul4(lay, a, w, out, gated=gated)
    assert torch.equal(first, out), "two equal calls differ"
    assert ctx.device_status() == B.STRATA_OK
    return out


def narrow(kind, gated, channels, stride, first):
    """Rows of out that start on fewer than 16 bytes, and what lies around them."""
    parts = 2 if gated else 1
    ctx, lay, a, w, _ = t.matmul_case(410, 2, 1, 96, parts * channels, gated, kind, 3)
    buf = torch.full((a.rows * stride + 8,), 99.0, dtype=torch.bfloat16, device=DEV)
    view = buf[first:first + a.rows * stride].view(a.rows, stride)[:, :channels]
    ctx.expert_matmul4(lay, a, w, view, gated=gated)
    t.check_products(lay, a, w, view, gated)
    view.fill_(99.0)
    assert bool((buf == 99.0).all()), "something beside the rows was written"
    assert ctx.device_status() == B.STRATA_OK
    return view


def scales(kind, gated):
    """One block of every row and one of every channel are not zero, and every scale differs from its neighbours': a product is not
    zero only where the two blocks meet, and is then one block's sum times two scales."""
    rows, inner, n = 700, 1056, ref.BLOCK[kind]
    half = 320
    ctx, lay, a, w, out = t.matmul_case(rows, 1, 1, inner, half * (2 if gated else 1), gated, kind, 6, spread=6)
    a.codes.zero_()
    w.codes.zero_()
    for q, where in ((a.codes, lambda i: i), (w.codes[0], lambda i: (i % half) * 5)):
        for i in range(q.shape[0]):
            at = where(i) % (inner // n) * (n // 2)
            q[i, at:at + n // 2] = 0x22                                # values 1
    ctx.expert_matmul4(lay, a, w, out, gated=gated)
    t.check_products(lay, a, w, out, gated)
    meet = (torch.arange(rows)[:, None] - 5 * torch.arange(half)[None]) % (inner // n) == 0
    assert bool((out.cpu() != 0)[~meet].any()) is False and bool((out.cpu() != 0)[meet].float().mean() > 0.9)
    assert ctx.device_status() == B.STRATA_OK
    return out


def capacity(kind, gated):
    ctx, lay, a, w, out = t.matmul_case(240, 4, 2, 128, 96, gated, kind, 5, R=2, slot_capacity=150)
    ctx.expert_matmul4(lay, a, w, out, gated=gated)
    t.check_products(lay, a, w, out, gated, count=np.full(4, 300))
    assert ctx.device_status() == B.STRATA_OK
    return out


def timeout(L):
    """The first load of one launch is expected to bring 16 bytes more than it does (see rows4_timeout_child.py)."""
    hook = L.strata_test_inject_short_load4
    hook.argtypes, hook.restype = [ctypes.c_int], None
    ctx, lay, a, w, out = t.matmul_case(1400, 2, 1, 2048, 1024, False, "nvfp4", 7)

    def call():
        ctx.expert_matmul4(lay, a, w, out)
        return out.clone()
    want = call()
    res = {"before": ctx.device_status()}
    hook(1)
    call()
    res["after_injection"] = ctx.device_status()
    res["header_words"] = ctx.workspace[:44].view(torch.int32).cpu().tolist()
    res["same_afterwards"] = bool(torch.equal(call(), want))
    res["after_normal_call"] = ctx.device_status()
    res["tile"] = L.strata_test_last_tile4()
    return res


def main(tile, what=""):
    L = B.lib()
    L.strata_test_tile4.argtypes, L.strata_test_tile4.restype = [ctypes.c_int], None
    L.strata_test_last_tile4.restype = ctypes.c_int
    L.strata_test_tile4(tile)
    if what == "timeout":
        print(json.dumps(timeout(L)), flush=True)
        return
    res = {}

    def run(name, f, *args):
        try:
            out = f(*args)
            if tile >= 0:
                assert L.strata_test_last_tile4() == tile
            res[name] = ["ok", hashlib.sha256(out.contiguous().view(torch.int16).cpu().numpy().tobytes()).hexdigest()[:16]]
        except B.StrataError as e:
            res[name] = ["refused" if e.code == B.STRATA_ERR_CUDA else repr(e), ""]
        except AssertionError as e:
            res[name] = [repr(e)[:400], ""]
    if tile < 0:                                                       # what the library chooses for few and for many rows, on a whole GPU
        for name, c in (("few", dict(tokens=8, E=8, K=2, inner=512, channels=512)),
                        ("many", dict(tokens=1536, E=2, K=1, inner=7168, channels=4096))):
            for kind in t.KINDS:
                run(f"{name}-{kind}", product, c, kind, False)
                res[f"{name}-{kind}"].append(L.strata_test_last_tile4())
    else:
        for kind in t.KINDS:
            for gated in (False, True):
                end = f"-{kind}-{'gated' if gated else 'plain'}"
                for name, c in SHAPES.items():
                    run(name + end, product, c, kind, gated)
                for i, n in enumerate(NARROW):
                    run(f"narrow{i}" + end, narrow, kind, gated, *n)
                run("scales" + end, scales, kind, gated)
                run("capacity" + end, capacity, kind, gated)
    print(json.dumps(res), flush=True)


if __name__ == "__main__":
    main(int(sys.argv[1]), *sys.argv[2:])
