"""Attention of many requests in one call: more than a warp has lanes, more than a block of
any of the kernels has threads, ended ones among them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.paged_util import Step
from tests.test_gpu_paged import _check

pytestmark = pytest.mark.gpu


def _lengths(batch, most, seed):
    rng = np.random.default_rng(seed)
    ctx, new = rng.integers(0, 90, batch), rng.integers(0, most + 1, batch)
    ended = rng.random(batch) < 0.2
    ctx[ended], new[ended] = 0, 0
    ctx[batch // 2], new[batch - 1] = 700, most
    return ctx.tolist(), new.tolist()


# few rows; 4 bands; 2 bands; 128 rows a tile; fp32 with tiles of 16 and of 64 rows
@pytest.mark.parametrize("dtypes,heads,kv,most", [
    (("f16", "bf16"), 4, 2, 2), (("f16",), 24, 1, 1), (("bf16",), 40, 1, 2), (("f16",), 64, 1, 3), (("f32",), 4, 2, 2),
    (("f32",), 32, 1, 2)])
@pytest.mark.parametrize("batch", [32, 33, 161, 321, 700])
@pytest.mark.parametrize("window", [0, 37])
def test_many_requests(dtypes, heads, kv, most, batch, window):
    for dtype in dtypes:
        _check(Step(*_lengths(batch, most, batch + heads), heads, kv, 64, 16, dtype, seed=batch), window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_with_a_long_one(dtype):
    """Cut tiles among many requests."""
    ctx, new = _lengths(200, 1, 3)
    ctx[77], new[77] = 20000, 3
    _check(Step(ctx, new, 4, 1, 128, 64, dtype, seed=8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_masked(dtype):
    ctx, new = _lengths(170, 9, 5)
    step = Step(ctx, new, 8, 2, 64, 8, dtype, seed=6)
    mask = torch.rand(step.rows, 9, generator=torch.Generator().manual_seed(1)) < 0.4
    mask[::5] = False
    _check(step, mask=mask)
