"""A role that gives up while the loading warp has nothing left to do: what a CTA has under way
ends before it does, the status says what happened, and the cache goes on working."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged
from tests.paged_util import Step

pytestmark = pytest.mark.gpu


# the tiles of a piece all fit the ring: 4 bands, 2 bands, one slot's rows, both slots'; few rows
@pytest.mark.parametrize("heads,kv,new,batch", [(24, 1, 1, 1), (40, 1, 1, 1), (4, 1, 25, 2), (40, 40, 130, 4), (8, 2, 3, 2)])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("chunk", [0, 1])
def test_giving_up_after_the_last_load(heads, kv, new, batch, hd, chunk):
    lib = cllm.load()
    lib.cllm_test_hold_paged.argtypes = [ctypes.c_void_p, ctypes.c_int]
    step = Step([230 - new] * batch, [new] * batch, heads, kv, hd, 32, "f16", seed=new)
    cache = paged.PagedCache(step.k, step.v, heads)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=32)
    want = cache.attention(0, step.q, rows, tables)
    cache.check()
    for _ in range(3):
        assert lib.cllm_test_hold_paged(cache._h, chunk) == 0
        cache.attention(0, step.q, rows, tables)
        assert lib.cllm_test_hold_paged(cache._h, -1) == 0
        with pytest.raises(cllm.CllmError) as e:
            cache.check()
        assert e.value.status == -5
        assert torch.equal(cache.attention(0, step.q, rows, tables), want)
        cache.check()
