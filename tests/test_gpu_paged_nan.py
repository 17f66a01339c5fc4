"""Infinities and NaN among the scores that a row does see: the row is NaN, and so is
its log-sum-exp, whichever kernel takes it and wherever its keys are cut (warps,
bands, slots, parts of a tile)."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged
from tests.paged_util import Step

pytestmark = pytest.mark.gpu

# (types, heads, key/value heads, cached tokens, new tokens, keys [0, this) that are NaN): one
# of a row's shares of the keys has nothing but NaN, the others have none
F16, F32 = ("bf16", "f16"), ("f32",)
SHARES = [
    (F16, 8, 2, [20], [3], 16),              # few rows: a warp's 16 keys
    (F16, 8, 2, [20, 150], [3, 2], 64),      # the whole first chunk
    (F16, 4, 4, [70], [30], 16),             # two tiles of few rows
    (F16, 8, 2, [9000], [3], 512),           # cut: whole parts
    (F16, 24, 1, [200], [1], 32),            # four bands: one band's keys
    (F16, 24, 1, [9000], [1], 1024),
    (F16, 40, 1, [200], [1], 64),            # two bands
    (F16, 40, 1, [9000], [1], 1024),
    (F16, 4, 1, [300], [25], 128),           # one slot's chunk
    (F16, 4, 1, [9000], [25], 1024),
    (F16, 40, 40, [300] * 4, [130] * 4, 128),    # 128 rows in each slot
    (F16, 40, 40, [8300] * 4, [130] * 4, 1024),
    (F32, 8, 2, [20], [3], 16), (F32, 8, 2, [9000], [3], 512),
    (F32, 8, 2, [200], [30], 64), (F32, 8, 2, [9000], [30], 512),
]
CASES = [(t, *c[1:]) for c in SHARES for t in c[0]]


def _call(step):
    cache = paged.PagedCache(step.k, step.v, step.heads)
    lse = torch.full((step.rows, step.heads), 7.0, device="cuda")
    got = cache.attention(step.layer, step.q, paged.PageRows(step.row_start, step.seq_len),
                          paged.PageTables(step.table, page_size=step.page), lse=lse)
    cache.check()
    return got, lse


@pytest.mark.parametrize("dtype,heads,kv,ctx,new,bad", CASES)
@pytest.mark.parametrize("hd", [64, 128])
def test_keys_of_nan_make_the_row_nan(dtype, heads, kv, ctx, new, bad, hd):
    step = Step(ctx, new, heads, kv, hd, 16 if ctx[0] < 1000 else 256, dtype, seed=bad)
    for b in range(len(ctx)):
        for pos in range(0, bad, step.page):
            page = int(step.table[b, pos // step.page])
            step.k[0, page, :, :min(step.page, bad - pos)] = math.nan
    got, lse = _call(step)
    assert bool(torch.isnan(got).all())
    assert bool(torch.isnan(lse).all())


@pytest.mark.parametrize("dtype,heads,kv,ctx,new,bad", [c for c in CASES if len(c[3]) == 1])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_query_that_is_no_number(dtype, heads, kv, ctx, new, bad, value):
    """One row's queries: that row is NaN, the others are what they are without."""
    step = Step(ctx, new, heads, kv, 64, 16 if ctx[0] < 1000 else 256, dtype, seed=bad + 1)
    o, want_lse, ab, delta = step.attention()
    tol, ltol = step.bound(ab, delta, o)
    r = step.rows // 2
    step.q[r] = value  # (with an infinity products of both signs meet)
    got, lse = _call(step)
    assert bool(torch.isnan(got[r]).all()) and bool(torch.isnan(lse[r]).all())
    rest = [i for i in range(step.rows) if i != r]
    assert bool(((got.double() - o).abs()[rest] <= tol[rest]).all())
    assert bool(((lse.double() - want_lse).abs()[rest] <= ltol[rest]).all())
