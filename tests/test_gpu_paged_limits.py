"""The paged cache at the ends of its sizes' ranges."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged
from tests.test_gpu_paged import _i32

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


def _none(t, value):
    """Whether all of a large tensor is `value`."""
    return all(bool((t[i:i + (1 << 28)] == value).all()) for i in range(0, t.numel(), 1 << 28))


def test_plan_of_the_most_rows():
    tables, rows = paged.PageTables.empty(8, 16, 2, 4), paged.PageRows.empty(2, 1)
    z = dict(device="cuda")
    slots, positions = torch.full((MOST,), 7, dtype=torch.int64, **z), torch.full((MOST,), 7, dtype=torch.int32, **z)
    rows = paged.PageRows(rows.row_start, rows.seq_len, rows.granted, slots, positions)
    paged.plan(tables, rows, _i32([0, 0]), _i32([3, 2]))
    torch.cuda.synchronize()
    assert rows.row_start.tolist() == [0, 3, 5] and rows.granted.tolist() == [1, 1]
    assert slots[:6].tolist() == [0, 1, 2, 16, 17, -1] and positions[:6].tolist() == [0, 1, 2, 0, 1, 0]
    assert _none(slots[5:], -1) and _none(positions[5:], 0)


@pytest.mark.parametrize("in_place", [True, False])
def test_plan_of_the_widest_table(in_place):
    z = dict(dtype=torch.int32, device="cuda")
    ring, held = torch.arange(8, **z), torch.zeros(1, **z)
    tables = paged.PageTables(torch.full((1, MOST), -1, **z), held, ring, _i32([0, 8, 0, 0]), 1)
    out = tables
    if not in_place:
        out = paged.PageTables(torch.full((1, MOST), 7, **z), torch.zeros(1, **z), ring, _i32([0, 0, 0, 0]), 1)
    rows = paged.PageRows.empty(1, 4)
    paged.plan(tables, rows, _i32([1]), _i32([2]), out=out)
    torch.cuda.synchronize()
    assert out.held.tolist() == [3] and out.state.tolist() == [3, 5, 0, 0]
    assert rows.slots.tolist() == [1, 2, -1, -1] and out.table[0, :4].tolist() == [0, 1, 2, -1]
    assert _none(out.table[0, 3:], -1)
