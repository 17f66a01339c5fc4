"""Calls on a paged cache go to the cache's device: on one that does not exist they fail and
leave everything as it was."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged
from tests.paged_util import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads,kv", [(4, 2), (40, 1)])
def test_calls_select_the_caches_device(dtype, heads, kv):
    lib = cllm.load()
    lib.cllm_test_paged_device.argtypes = [ctypes.c_void_p, ctypes.c_int]
    assert lib.cllm_test_paged_device(None, 0) == -1
    step = Step([40], [3], heads, kv, 64, 16, dtype)
    cache = paged.PagedCache(step.k, step.v, heads)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    out, before = torch.full_like(step.q, 5.0), step.k.clone()
    k, slots = torch.ones(3, kv, 64, device="cuda", dtype=step.q.dtype), torch.arange(3, device="cuda")
    here = lib.cllm_test_paged_device(cache._h, torch.cuda.device_count())
    assert here == torch.cuda.current_device()
    try:
        for call in (lambda: cache.attention(0, step.q, rows, tables, out=out), lambda: cache.append(0, k, k, slots), cache.check):
            with pytest.raises(cllm.CllmError) as e:
                call()
            assert e.value.status == -3
    finally:
        assert lib.cllm_test_paged_device(cache._h, here) == torch.cuda.device_count()
    torch.cuda.synchronize()
    assert torch.cuda.current_device() == here
    assert bool((out == 5.0).all())
    assert torch.equal(step.k.nan_to_num(9.0), before.nan_to_num(9.0))
    cache.attention(0, step.q, rows, tables, out=out)
    cache.check()
    assert bool(torch.isfinite(out).all()) and not bool((out == 5.0).all())
