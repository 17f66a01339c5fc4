"""Calls on a stream that is not the current one."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged
from tests.paged_util import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_an_allocated_output_belongs_to_the_stream_that_writes_it(dtype):
    """Memory freed on the current stream may still be read there: the call does not take it."""
    step = Step([200], [40], 8, 2, 128, 16, dtype, seed=1)
    cache = paged.PagedCache(step.k, step.v, 8)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    want = cache.attention(0, step.q, rows, tables)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    freed = torch.empty_like(step.q)
    address = freed.data_ptr()
    del freed
    got = cache.attention(0, step.q, rows, tables, stream=side)
    assert got.data_ptr() != address
    assert torch.empty_like(step.q).data_ptr() == address  # (the current stream still has it)
    cache.check(side)
    assert torch.equal(got, want)
