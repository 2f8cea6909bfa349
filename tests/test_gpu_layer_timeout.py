"""The time-out path of the layer kernels' bounded waits (STRATA_ERR_TIMEOUT), exercised without faulting the GPU, in a child
process that loads the test-hooks build (see test_gpu_timeout.py)."""
import json
import os
import subprocess
import sys

import pytest

from paper_2607_26444_b200 import binding as B
from paper_2607_26444_b200 import build as strata_build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kind", ["matmul", "norm_grad", "norm_grad_warp"])
def test_a_wait_that_runs_out_reports_timeout_and_the_context_recovers(kind):
    env = dict(os.environ, STRATA_MOE_LIB=strata_build.build_test_hooks())
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "layer_timeout_child.py"), kind], env=env,
                       capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-3000:]
    res = json.loads([l for l in r.stdout.splitlines() if l.startswith("{")][-1])
    assert res["status_before"] == B.STRATA_OK
    assert res["status_after_injection"] == B.STRATA_ERR_TIMEOUT
    assert res["status_read_again"] == B.STRATA_OK
    assert res["header_words_after_recovery"] == [0] * 10
    assert res["same_afterwards"] and res["status_after_normal_call"] == B.STRATA_OK
