"""Page plans of every number of requests up to the limit, each the first call of its process
(a kernel's shared-memory limit, once raised, stays raised)."""
import os
import subprocess
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged
from tests.paged_util import TablesModel
from tests.test_gpu_paged import _i32, _same

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def plan_once(batch):
    rng = np.random.default_rng(batch)
    tables, rows = paged.PageTables.empty(3 * batch, 8, batch, 5), paged.PageRows.empty(batch, 10 * batch)
    model = TablesModel(3 * batch, 8, batch, 5)
    for _ in range(2):
        ctx, new = rng.integers(0, 12, batch).tolist(), rng.integers(0, 10, batch).tolist()
        ctx = [min(c, 8 * len(t)) for c, t in zip(ctx, model.tables)]
        paged.plan(tables, rows, _i32(ctx), _i32(new))
        _same(tables, rows, model, model.plan(ctx, new, 10 * batch), batch)


@pytest.mark.parametrize("batch", [2450, 2451, 2457, 2458, 4096])
def test_plan_of_many_requests_is_a_process_first_call(batch):
    code = f"from tests.test_gpu_paged_plan_sizes import plan_once; plan_once({batch})"
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
