"""Each of the four tiles of the 4-bit products by itself, over both kinds, plain and gated: odd row counts, partial channel tiles,
inner extents that end inside a span, every scale at its block, rows of out on 16, 8, 4 and 2 bytes.  The library chooses tiles by
an estimate; the test-hooks build takes the one that the test names (rows4_tiles_child.py, tolerances of test_gpu_rows4.py)."""
import functools
import json
import os
import subprocess
import sys

import pytest
import torch

from paper_2607_26444_b200 import binding as B
from paper_2607_26444_b200 import build as strata_build

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
import test_gpu_rows4 as rows4  # noqa: E402

ROOT = os.path.dirname(HERE)
pytestmark = pytest.mark.gpu
TILES = ["1x1x64", "1x2x96", "2x1x192", "2x2x192"]               # CTAs, blocks of 128 channels, rows


@functools.cache
def child(tile, *what):
    env = dict(os.environ, STRATA_MOE_LIB=strata_build.build_test_hooks())
    r = subprocess.run([sys.executable, os.path.join(HERE, "rows4_tiles_child.py"), str(tile), *what], env=env, capture_output=True, text=True,
                       timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads([line for line in r.stdout.splitlines() if line.startswith("{")][-1])


@pytest.mark.parametrize("tile", range(4), ids=TILES)
def test_every_shape_on_each_tile(tile):
    """A tile refuses what it cannot do: gate and up by eights where gated channels are no multiple of 16 (one block of channels), more
    experts than its tables hold (the widest)."""
    res = child(tile)
    assert len(res) == 2 * 2 * 17
    for name, (what, _) in res.items():
        by_eights = tile in (0, 2) and name.endswith("gated") and name.split("-")[0] in ("odd", "narrow2", "narrow3", "narrow4", "narrow5")
        too_many = tile == 3 and name.startswith("too_many")
        assert what == ("refused" if by_eights or too_many else "ok"), (name, what)


def test_all_tiles_give_the_same_bits():
    """Each sums a row's values in the same order, 64 at a time, so that neither the estimate nor a budget of SMs shows in the results."""
    for name in child(1):
        bits = {child(tile)[name][1] for tile in range(4) if child(tile)[name][0] == "ok"}
        assert len(bits) == 1, (name, [child(tile)[name] for tile in range(4)])


def test_few_and_many_rows_take_different_tiles():
    """On a whole GPU the widest tile is what many rows of a long product get, without being asked for."""
    res = child(-1)
    assert all(v[0] == "ok" for v in res.values()), res
    assert res["few-mxfp4"][2] in (0, 1) and res["few-nvfp4"][2] in (0, 1)
    if torch.cuda.get_device_properties(0).multi_processor_count == 148:
        assert res["many-mxfp4"][2] == 3 and res["many-nvfp4"][2] == 3


def test_a_wait_of_the_widest_tile_that_runs_out():
    res = child(3, "timeout")
    assert res["tile"] == 3 and res["before"] == B.STRATA_OK and res["after_injection"] == B.STRATA_ERR_TIMEOUT
    assert res["header_words"] == [0] * 11 and res["same_afterwards"] and res["after_normal_call"] == B.STRATA_OK


def test_the_widest_tile_captured_and_on_two_streams():
    """Two contexts whose products take the widest tile, each in a graph, replayed at once on new codes."""
    cases = []
    for kind, seed in (("mxfp4", 1), ("nvfp4", 2)):
        ctx, lay, a, w, out = rows4.matmul_case(1536, 2, 1, 7168, 4096, False, kind, seed)
        call = functools.partial(ctx.expert_matmul4, lay, a, w, out)
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        a.codes.copy_(a.codes.flip(0).contiguous())
        cases.append((ctx, call, out, graph))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        for stream, case in zip(streams, cases):
            with torch.cuda.stream(stream):
                case[3].replay()
    torch.cuda.synchronize()
    for ctx, call, out, _ in cases:
        got = out.clone()
        call()
        assert torch.equal(out, got) and not bool((got == 99.0).any()) and ctx.device_status() == B.STRATA_OK
