"""4-bit rows on the GPU: quantiser, its inverse and the experts' products against 64-bit implementations (rows4_reference.py).

Tolerances, derived before the first run:
- codes, block scales and row scales of the quantiser: equal (the reference decides ties exactly; a row scale is one binary32
  division);
- values: code * (block * row scale), two binary32 roundings (2^-23) and one to bf16 (half an ulp); mxfp4 in fp32 exactly;
- products: the matrix unit sums in binary32 storage with at least 13 fraction bits kept in each alignment: 2^-13 * sum|a w|, a
  few binary32 roundings (2^-18 relative), half a bf16 ulp; gated as in test_gpu_layer.py."""
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
KINDS = ["mxfp4", "nvfp4"]


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def bits(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def half_ulp(a):
    return np.ldexp(1.0, np.maximum(np.frexp(a)[1], -125) - 9)


def context():
    return B.MoEContext(1, 1, 8, 1, 1)


def check_codes(x, q, kind):
    codes, block, scale = ref.quantize(f64(x), kind)
    assert np.array_equal(bits(q.block), block)
    assert np.array_equal(ref.unpack(bits(q.codes)), codes)
    if kind == "nvfp4":
        assert np.array_equal(q.scale.cpu().numpy().astype(np.float64), scale)


# ---- quantiser and its inverse ------------------------------------------------------------------------------------

SHAPES = [(1, 32), (2, 64), (3, 96), (5, 1024), (7, 1056), (33, 2048), (129, 7200), (4, 8192), (3, 16416), (2, 32768), (2100, 2048)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_quantize_codes_and_scales(rows, cols, kind):
    g = gen(rows + cols)
    wide = (randn(g, rows, cols + 24) * torch.exp(2 * randn(g, rows, 1))).to(torch.bfloat16)
    for x in (wide[:, :cols], wide[:, :cols].contiguous()):
        q = B.empty_rows4((rows,), cols, kind)
        ctx = context()
        ctx.quantize_rows4(x, q)
        check_codes(x, q, kind)
    out, out32 = torch.empty_like(x), torch.empty((rows, cols), device=DEV)
    ctx.dequantize_rows4(q, out)
    ctx.dequantize_rows4(q, out32)
    want = ref.values(bits(q.codes), bits(q.block), kind, None if q.scale is None else f64(q.scale))
    assert np.all(np.abs(f64(out32) - want) <= (0 if kind == "mxfp4" else 2.0 ** -23) * np.abs(want))
    assert np.all(np.abs(f64(out) - want) <= half_ulp(want) + 2.0 ** -23 * np.abs(want))


@pytest.mark.parametrize("kind", KINDS)
def test_quantize_ties_and_signs(kind):
    """Every multiple of 1/8 up to 8 under a known largest magnitude: half-way cases go to the even code, signs stay."""
    grid = torch.arange(-64, 64, device=DEV, dtype=torch.float32) / 8
    for top in (4.0, 6.0, 6.75, 7.0, 7.96875):
        x = grid.clamp(-top, top).reshape(-1, 16)
        rows = torch.cat((x, torch.full((x.shape[0], 16), top, device=DEV)), dim=1).to(torch.bfloat16)
        for power in (-20, 0, 13):
            r = (rows.float() * 2.0 ** power).to(torch.bfloat16)
            q = B.empty_rows4((r.shape[0],), 32, kind)
            context().quantize_rows4(r, q)
            check_codes(r, q, kind)


@pytest.mark.parametrize("kind", KINDS)
def test_quantize_every_pair_of_magnitudes(kind):
    """All 128 fractions against all 128 as the row's largest (and the block's): every quotient that bf16 values can form."""
    a = (torch.arange(128, 256, device=DEV).float() / 128).to(torch.bfloat16)
    for low in (1.0, 0.5, 0.25, 0.125, 0.0625):
        x = torch.empty((128, 160), dtype=torch.bfloat16, device=DEV)
        x[:, :128] = (a.float() * low).to(torch.bfloat16)[None]
        x[:, 128:] = a[:, None]                                        # the row's largest, in a block of its own
        x[:, 127:128] = a[:, None] if kind == "mxfp4" else x[:, 127:128]
        q = B.empty_rows4((128,), 160, kind)
        context().quantize_rows4(x, q)
        check_codes(x, q, kind)


@pytest.mark.parametrize("kind", KINDS)
def test_quantize_extremes(kind):
    x = torch.zeros((8, 64), dtype=torch.bfloat16, device=DEV)
    small = torch.tensor([1.0, -0.5, 3.0, 0.25], device=DEV).repeat(8)
    x[1, :32] = (small * 2.0 ** -126).to(torch.bfloat16)               # zeros beside the smallest normal numbers
    x[2, :] = (small.repeat(2) * 2.0 ** -131).to(torch.bfloat16)       # subnormal numbers
    x[3, :] = torch.finfo(torch.bfloat16).max
    x[4, 40] = -torch.finfo(torch.bfloat16).max
    x[4, :32] = 1.0                                                    # blocks far below the row's largest
    x[5, 0] = 1.0
    x[6, :32], x[6, 32:] = 448.0, 2.0 ** -10                           # a block scale below the least of e4m3
    x[7, :] = -0.0
    q = B.empty_rows4((8,), 64, kind)
    ctx = context()
    ctx.quantize_rows4(x, q)
    codes, block, scale = ref.quantize(f64(x), kind)
    assert np.array_equal(bits(q.block), block)
    assert np.array_equal(ref.unpack(bits(q.codes)), codes)
    if kind == "nvfp4":                                                # subnormal row scales: rounded to what binary32 holds there
        assert np.array_equal(q.scale.cpu().numpy().astype(np.float64), scale)
    out = torch.empty((8, 64), device=DEV)
    ctx.dequantize_rows4(q, out)
    want = ref.values(bits(q.codes), bits(q.block), kind, None if q.scale is None else f64(q.scale))
    assert np.all(np.abs(f64(out) - want) <= 2.0 ** -23 * np.abs(want) + 2.0 ** -149)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_quantize_not_finite(bad):
    """mxfp4: the block stands for NaN; nvfp4: the row does.  What else there is stays as it is."""
    g = gen(4)
    x = randn(g, 3, 96).to(torch.bfloat16)
    clean = x.clone()
    x[1, 40] = bad
    ctx = context()
    for kind in KINDS:
        q, c = B.empty_rows4((3,), 96, kind), B.empty_rows4((3,), 96, kind)
        out, want = torch.empty_like(x), torch.empty_like(x)
        ctx.quantize_rows4(x, q)
        ctx.dequantize_rows4(q, out)
        ctx.quantize_rows4(clean, c)
        ctx.dequantize_rows4(c, want)
        hit = torch.zeros((3, 96), dtype=torch.bool, device=DEV)
        hit[1, slice(32, 64) if kind == "mxfp4" else slice(None)] = True
        assert bool(torch.isnan(out[hit]).all()) and torch.equal(out[~hit], want[~hit])


def test_every_code_and_scale_byte_is_decoded():
    codes = torch.arange(256, device=DEV).to(torch.uint8).repeat(256, 1)                     # every pair of codes
    for kind in KINDS:
        n = 512 // ref.BLOCK[kind]
        block = torch.arange(256, device=DEV).to(torch.uint8)[:, None].repeat(1, n).contiguous()
        typed = block.view(torch.float8_e8m0fnu if kind == "mxfp4" else torch.float8_e4m3fn)
        out = torch.empty((256, 512), device=DEV)
        context().dequantize_rows4(B.Rows4(codes, typed), out)
        want = ref.values(codes.cpu().numpy(), block.cpu().numpy(), kind)
        got = f64(out)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        with np.errstate(over="ignore"):
            assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want.astype(np.float32).astype(np.float64)))


@pytest.mark.parametrize("kind", KINDS)
def test_rows_in_use_only_and_no_rows(kind):
    ctx = B.MoEContext(1, 20, 8, 4, 2, allow_unrouted=True)
    ids = torch.randint(0, 4, (1, 20, 2), device=DEV, dtype=torch.int32)
    ids[0, ::4] = -1
    lay = ctx.layout(ids)
    used = int(lay.expert_offset[4])
    x = randn(gen(8), 40, 64).to(torch.bfloat16)
    q = B.empty_rows4((40,), 64, kind)
    for t in (q.codes, q.block):
        t.view(torch.uint8).fill_(0x55)
    ctx.quantize_rows4(x, q, layout=lay)
    assert 0 < used < 40 and np.all(bits(q.codes)[used:] == 0x55) and np.all(bits(q.block)[used:] == 0x55)
    out = torch.full((40, 64), 99.0, dtype=torch.bfloat16, device=DEV)
    ctx.dequantize_rows4(q, out, layout=lay)
    assert bool((out[used:] == 99.0).all()) and not bool((out[:used] == 99.0).any())
    none = B.empty_rows4((0,), 64, kind)
    ctx.quantize_rows4(x[:0], none)
    ctx.dequantize_rows4(none, out[:0])
    assert ctx.device_status() == B.STRATA_OK


# ---- the experts' products ------------------------------------------------------------------------------------------

def random_rows4(g, shape, cols, kind, spread, level=0, pad=0):
    """Random codes and block scales around 2^level, `spread` binades up and down; rows `pad` bytes apart."""
    n = cols // ref.BLOCK[kind]
    codes = torch.full((*shape, cols // 2 + pad), 0xEE, dtype=torch.uint8, device=DEV)
    codes[..., :cols // 2] = torch.randint(0, 256, (*shape, cols // 2), generator=g, device=DEV).to(torch.uint8)
    block = torch.full((*shape, (n + 15) // 16 * 16 + pad), 0xEE, dtype=torch.uint8, device=DEV)
    if kind == "mxfp4":
        block[..., :n] = (127 + level + torch.randint(-spread, spread + 1, (*shape, n), generator=g, device=DEV)).to(torch.uint8)
        return B.Rows4(codes[..., :cols // 2], block.view(torch.float8_e8m0fnu)[..., :n])
    e = torch.randint(-spread, spread + 1, (*shape, n), generator=g, device=DEV).clamp(-6, 8)
    block[..., :n] = (8 * (7 + e) + torch.randint(0, 7, (*shape, n), generator=g, device=DEV)).to(torch.uint8)
    scale = (0.5 + torch.rand(shape, generator=g, device=DEV)) * 2.0 ** level
    return B.Rows4(codes[..., :cols // 2], block.view(torch.float8_e4m3fn)[..., :n], scale)


def matmul_case(tokens, E, K, inner, channels, gated, kind, seed, R=1, skew=False, pad=0, spread=2, **ctx_kw):
    g = gen(seed)
    ctx = B.MoEContext(R, tokens, 8, E, K, **ctx_kw)
    keys = torch.rand((R * tokens, E), generator=g, device=DEV)
    if skew:                                                       # most tokens want the first experts; some get none
        keys = keys * (1 + torch.arange(E, device=DEV)) ** 2
    ids = torch.argsort(keys, dim=1)[:, :K].to(torch.int32).reshape(R, tokens, K).contiguous()
    if ctx_kw.get("allow_unrouted"):
        ids[:, ::3] = -1
    lay = ctx.layout(ids)
    a = random_rows4(g, (ctx.recv_rows,), inner, kind, spread, -2, pad)
    w = random_rows4(g, (E, channels), inner, kind, spread, -2 - int(np.log2(inner) / 2))
    out = torch.full((ctx.recv_rows, channels // 2 if gated else channels), 99.0, dtype=torch.bfloat16, device=DEV)
    return ctx, lay, a, w, out


def plain(q):
    scale = None if q.scale is None else f64(q.scale)
    return ref.values(bits(q.codes), bits(q.block), "mxfp4" if q.type == B.STRATA_T_MXF4 else "nvfp4", scale)


def check_products(lay, a, w, out, gated, count=None):
    count = lay.expert_count.cpu().numpy() if count is None else count
    offset = lay.expert_offset.cpu().numpy()
    got, seen = f64(out), np.zeros(out.shape[0], bool)
    av, wv = plain(a), plain(w)
    half = wv.shape[1] // 2
    for e in range(wv.shape[0]):
        r = slice(int(offset[e]), int(offset[e]) + int(count[e]))
        seen[r] = True
        y, mag = av[r] @ wv[e].T, np.abs(av[r]) @ np.abs(wv[e]).T
        rel = 2.0 ** -18
        if gated:
            gate, up, gm, um = y[:, :half], y[:, half:], mag[:, :half], mag[:, half:]
            with np.errstate(over="ignore"):
                s = gate / (1 + np.exp(-gate))
            y, mag, rel = s * up, 1.1 * gm * np.abs(up) + np.abs(s) * um, rel * (1 + np.abs(gate))
        bad = ~(np.abs(got[r] - y) <= half_ulp(y) + rel * np.abs(y) + 2.0 ** -13 * mag + 1e-30)
        assert not bad.any(), (e, int(bad.sum()), got[r][bad][:4], y[bad][:4], np.argwhere(bad)[:4])
    assert np.all(got[~seen] == 99.0)                              # rows of no segment are not written


MATMULS = [
    dict(tokens=1, E=8, K=1, inner=32, channels=4),                   # one row, the least of everything
    dict(tokens=1, E=32, K=8, inner=512, channels=256),               # one token
    dict(tokens=5, E=4, K=2, inner=160, channels=100),                # odd sizes below one tile
    dict(tokens=64, E=4, K=2, inner=256, channels=128),
    dict(tokens=100, E=3, K=3, inner=416, channels=132),              # 100 rows each
    dict(tokens=257, E=3, K=2, inner=1056, channels=260, skew=True),  # more than one row tile
    dict(tokens=700, E=7, K=2, inner=288, channels=388, skew=True),   # several row tiles, idle experts
    dict(tokens=33, E=300, K=4, inner=128, channels=64),              # more experts than SMs, most nearly empty
    dict(tokens=900, E=2, K=2, inner=128, channels=1028),
    dict(tokens=40, E=6, K=2, inner=256, channels=640, R=2, segment_align=16),
    dict(tokens=50, E=6, K=2, inner=256, channels=384, allow_unrouted=True),
    dict(tokens=2048, E=2, K=1, inner=64, channels=512),              # short inner extent, many tiles per CTA
    dict(tokens=3000, E=4, K=4, inner=32, channels=1200, skew=True),
    dict(tokens=45, E=5, K=2, inner=480, channels=274),               # an odd number of gated channels: rows of out on two bytes
    dict(tokens=300, E=3, K=2, inner=736, channels=510),
    dict(tokens=1300, E=3, K=2, inner=2304, channels=640),            # several stages round, three scale boxes
    dict(tokens=1500, E=2, K=1, inner=4128, channels=1056),           # long inner extent, many rows
    dict(tokens=8000, E=640, K=8, inner=64, channels=256),            # more experts than the widest tile has tables for
    dict(tokens=4000, E=520, K=8, inner=512, channels=96, skew=True),
]


@pytest.mark.parametrize("c", MATMULS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", KINDS)
def test_expert_matmul4_against_64_bits(c, gated, kind):
    ctx, lay, a, w, out = matmul_case(gated=gated, kind=kind, seed=41, pad=32, **c)
    ctx.expert_matmul4(lay, a, w, out, gated=gated)
    assert ctx.device_status() == B.STRATA_OK
    check_products(lay, a, w, out, gated)
    first = out.clone()
    ctx.expert_matmul4(lay, a, w, out, gated=gated)
    assert torch.equal(first, out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [40, 120, 700])
def test_every_scale_meets_its_block(kind, rows):
    """One block of one row and one of one channel are not zero: each scale is found where it belongs."""
    inner, channels, n = 1056, 300, ref.BLOCK[kind]
    ctx, lay, a, w, out = matmul_case(rows, 1, 1, inner, channels, False, kind, 6, spread=6)
    a.codes.zero_()
    w.codes.zero_()
    blocks = inner // n
    for r in range(rows):                                            # row r: block r % blocks; every channel: all blocks, values 1
        at = (r % blocks) * (n // 2)
        a.codes[r, at:at + n // 2] = 0x22
    w.codes.fill_(0x22)
    ctx.expert_matmul4(lay, a, w, out)
    check_products(lay, a, w, out, False)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", KINDS)
def test_expert_matmul4_fixed_capacity(gated, kind):
    ctx, lay, a, w, out = matmul_case(24, 4, 2, 128, 64, gated, kind, 5, R=2, slot_capacity=40)
    ctx.expert_matmul4(lay, a, w, out, gated=gated)
    assert ctx.device_status() == B.STRATA_OK
    check_products(lay, a, w, out, gated, count=np.full(4, 80))


def test_expert_matmul4_odd_channels_strides_and_scales():
    for channels, stride in ((131, 131), (1, 1), (128, 129)):
        ctx, lay, a, w, out = matmul_case(90, 3, 2, 128, channels, False, "nvfp4", 23)
        wide = torch.full((a.rows, stride), 99.0, dtype=torch.bfloat16, device=DEV)
        scales = torch.zeros((a.rows, 3), device=DEV)
        scales[:, 1] = a.scale
        scales[7] = 0
        a = B.Rows4(a.codes, a.block, scales[:, 1])
        ctx.expert_matmul4(lay, a, w, wide[:, :channels])
        check_products(lay, a, w, wide[:, :channels], False)
        assert bool((wide[:, channels:] == 99.0).all())
        bare = B.Rows4(a.codes, a.block), B.Rows4(w.codes, w.block)    # without scales of rows and channels
        ctx.expert_matmul4(lay, *bare, wide[:, :channels])
        check_products(lay, *bare, wide[:, :channels], False)


def test_rows_and_blocks_that_are_not_a_number_stay_apart():
    """A NaN scale (a row beside the segment, a row of its own) shows in its row alone."""
    ctx, lay, a, w, out = matmul_case(50, 6, 2, 256, 384, False, "mxfp4", 31, allow_unrouted=True)
    ctx.expert_matmul4(lay, a, w, out)
    want = out.clone()
    used = int(lay.expert_offset[6])
    a.block.view(torch.uint8)[used:] = 255
    a.block.view(torch.uint8)[3, 1] = 255
    ctx.expert_matmul4(lay, a, w, out)
    keep = torch.arange(a.rows, device=DEV) != 3
    assert bool(torch.isnan(out[3]).all()) and torch.equal(out[keep], want[keep])
    assert ctx.device_status() == B.STRATA_OK


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [30, 400])
def test_rows_of_out_that_start_on_fewer_than_16_bytes(rows, gated):
    """Every start of a row of out (16, 8, 4 and 2 bytes), with channels that end inside a piece; what lies around is left alone."""
    for channels in (96, 100, 102) if gated else (96, 100, 101):
        for stride, first in ((128, 0), (132, 0), (130, 0), (129, 0), (128, 4), (128, 2), (128, 1)):
            ctx, lay, a, w, out = matmul_case(rows, 3, 2, 96, channels, gated, "mxfp4", 3)
            wide = channels // 2 if gated else channels
            buf = torch.full((a.rows * stride + 8,), 99.0, dtype=torch.bfloat16, device=DEV)
            view = buf[first:first + a.rows * stride].view(a.rows, stride)[:, :wide]
            ctx.expert_matmul4(lay, a, w, view, gated=gated)
            check_products(lay, a, w, view, gated)
            around = buf.clone()
            around[first:first + a.rows * stride].view(a.rows, stride)[:, :wide] = 99.0
            assert bool((around == 99.0).all())
