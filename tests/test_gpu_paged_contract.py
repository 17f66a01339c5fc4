"""Calls of the paged cache that are refused because they would be answered with something
other than what was asked for."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged
from tests.paged_util import Step

pytestmark = pytest.mark.gpu


def _step(dtype="f16"):
    step = Step([20], [3], 4, 2, 64, 16, dtype)
    cache = paged.PagedCache(step.k, step.v, 4)
    return step, cache, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)


@pytest.mark.parametrize("shape", [(3, 0), (0,), (3,), (3, 1, 1)])
def test_a_mask_without_words_is_refused(shape):
    step, cache, rows, tables = _step()
    out = torch.full_like(step.q, 5.0)
    with pytest.raises(ValueError, match="block_mask"):
        cache.attention(0, step.q, rows, tables, out=out, block_mask=torch.zeros(shape, device="cuda", dtype=torch.int32))
    assert bool((out == 5.0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_output_over_the_queries_is_refused(dtype):
    """A row that is done again from the definition would read its own result."""
    step, cache, rows, tables = _step(dtype)
    before = step.q.clone()
    with pytest.raises(cllm.CllmError):
        cache.attention(0, step.q, rows, tables, out=step.q)
    assert torch.equal(step.q, before)
