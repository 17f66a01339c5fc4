"""A plan that refuses requests for want of rows, and the append and attention of its step:
the refused requests' rows are zeros, nothing is reported, the others are unharmed."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged
from tests.test_gpu_paged import _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,kv", [(4, 2), (40, 1), (64, 1)])
@pytest.mark.parametrize("new,max_rows,kept", [
    ([3, 7, 2, 5], 12, 3),          # the last one straddles the end
    ([3, 7, 2, 5, 0, 4], 8, 1),     # others lie wholly past it, one of them without rows
    ([3] * 40, 50, 16),             # more requests than a warp has lanes
    ([2, 2 ** 31 - 1, 4], 20, 1),   # row_start at its limit
    ([30], 20, 0)])
def test_refused_rows_are_zeros_and_no_error(dtype, heads, kv, new, max_rows, kept):
    batch, hd, page = len(new), 64, 8
    gen = torch.Generator(device="cuda").manual_seed(0)
    kp, vp = (torch.zeros(1, 64, kv, page, hd, device="cuda", dtype=dtype) for _ in range(2))
    cache = paged.PagedCache(kp, vp, heads)
    tables, rows = paged.PageTables.empty(64, page, batch, 8), paged.PageRows.empty(batch, max_rows)
    paged.plan(tables, rows, _i32([0] * batch), _i32(new))
    assert rows.granted.tolist() == [1] * kept + [0] * (batch - kept)
    live = sum(new[:kept])
    q = torch.randn(max_rows, heads, hd, device="cuda", generator=gen).to(dtype)
    k, v = (torch.randn(max_rows, kv, hd, device="cuda", generator=gen).to(dtype) for _ in range(2))
    cache.append(0, k, v, rows.slots)
    out, lse = torch.full_like(q, 5.0), torch.full((max_rows, heads), 5.0, device="cuda")
    cache.attention(0, q, rows, tables, out=out, lse=lse)
    cache.check()
    assert bool((out[live:] == 0).all()) and bool(torch.isneginf(lse[live:]).all())
    # the granted ones as in a step of their own
    if kept:
        alone = paged.PageRows(rows.row_start[:kept + 1].clone(), rows.seq_len[:kept].clone())
        want = cache.attention(0, q[:live].contiguous(), alone, tables)
        cache.check()
        u = torch.finfo(dtype).eps
        # (work may be cut in other places: each side rounds its probabilities and its result once)
        assert bool(((out[:live].double() - want.double()).abs() <= 4 * u * v.abs().max() + 1e-5).all())
