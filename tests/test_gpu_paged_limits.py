"""The paged cache at the ends of its sizes' ranges."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads", [1, 24, 40])
@pytest.mark.parametrize("length", [2 ** 31 - 8, 2 ** 31 - 8191])
def test_a_length_whose_chunks_pass_32_bits_is_reported(dtype, hd, heads, length):
    """The longest table, every entry the same page: nothing is read of a request that long."""
    page = 8
    k = torch.randn(1, 1, 1, page, hd, device="cuda").to(dtype)
    cache = paged.PagedCache(k, k.clone(), heads)
    table = torch.zeros(2, (2 ** 31 - 8) // page, dtype=torch.int32, device="cuda")
    q = torch.randn(2, heads, hd, device="cuda").to(dtype)
    out = torch.full_like(q, 5.0)
    cache.attention(0, q, paged.PageRows(_i32([0, 1, 2]), _i32([8, length])), paged.PageTables(table, page_size=page), out=out)
    with pytest.raises(cllm.CllmError) as e:
        cache.check()
    assert e.value.status == -6
    assert bool((out[1] == 0).all())
    want = torch.softmax(q[0].double() @ k[0, 0, 0].double().T * hd ** -0.5, -1) @ k[0, 0, 0].double()
    # (V is K: a probability's and the result's rounding, each of at most max |V|)
    assert bool(((out[0].double() - want).abs() <= 4 * torch.finfo(dtype).eps * k.abs().max().double() + 1e-5).all())
