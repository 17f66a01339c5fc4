"""Argument checks of the paged-cache calls that run before any CUDA call (CPU,
no GPU): only invalid inputs are passed, a valid one would go on to the device.
And the tests' own model of the page plan on a hand-worked step."""
import ctypes

import pytest

from paper_2403_00835_gb300 import cllm, paged
from tests.paged_util import TablesModel
from tests.test_abi import declared_functions

EINVAL, EUNSUPPORTED = -1, -8
P = 0x1000  # never dereferenced: the checks fail first


@pytest.fixture(scope="module")
def lib():
    return paged.load()


def test_every_call_is_bound_and_exported(lib):
    assert set(paged.EXPORTS) <= set(declared_functions())
    assert all(hasattr(lib, n) for n in paged.EXPORTS)


def _desc(**kw):
    a = dict(k=P, v=P, dtype=cllm.CLLM_BF16, layers=2, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, n_heads=4,
             stride_layer=8 * 16 * 2 * 64, stride_page=16 * 2 * 64, stride_head=16 * 64, stride_pos=64)
    a.update(kw)
    return paged._Desc(*[a[f] for f, _ in paged._Desc._fields_])


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=P + 8), EINVAL), (dict(dtype=3), EINVAL), (dict(layers=0), EINVAL),
    (dict(n_pages=0), EINVAL), (dict(page_size=0), EINVAL), (dict(n_heads=0), EINVAL), (dict(stride_pos=32), EINVAL),
    (dict(stride_head=1028), EINVAL), (dict(stride_page=-2048), EINVAL), (dict(head_dim=96), EUNSUPPORTED),
    (dict(page_size=24), EUNSUPPORTED), (dict(page_size=4), EUNSUPPORTED), (dict(page_size=512), EUNSUPPORTED),
    (dict(n_heads=5), EUNSUPPORTED), (dict(n_heads=130), EUNSUPPORTED)])
def test_create_refuses(lib, kw, want):
    h = ctypes.c_void_p()
    assert lib.cllm_paged_create(ctypes.byref(_desc(**kw)), ctypes.byref(h)) == want
    assert not h.value


def test_null_caches(lib):
    assert lib.cllm_paged_create(None, None) == EINVAL
    lib.cllm_paged_destroy(None)  # no-op
    assert lib.cllm_paged_status(None, None) == EINVAL
    zeros = ctypes.create_string_buffer(256)
    assert lib.cllm_paged_append(None, ctypes.addressof(zeros), None) == EINVAL
    assert lib.cllm_paged_attention(None, ctypes.addressof(zeros), None) == EINVAL


def _plan(lib, B=2, ctx=P, new=P, other=None, rows=None, **kw):
    t = dict(table=P, held=P, ring=P, state=P, max_batch=4, width=8, n_pages=16, page_size=16)
    t.update(kw)
    a = paged._Tables(*[t[f] for f, _ in paged._Tables._fields_])
    t.update(other or {})
    b = paged._Tables(*[t[f] for f, _ in paged._Tables._fields_])
    r = dict(row_start=P, seq_len=P, granted=P, slots=P, positions=P, max_rows=32)
    r.update(rows or {})
    r = paged._Rows(*[r[f] for f, _ in paged._Rows._fields_])
    return lib.cllm_page_plan(ctypes.addressof(a), ctypes.addressof(b), ctypes.addressof(r), B, ctx, new, None)


@pytest.mark.parametrize("kw", [
    dict(B=-1), dict(B=5), dict(ctx=None), dict(new=None), dict(table=None), dict(held=None), dict(ring=None), dict(state=None),
    dict(max_batch=0), dict(max_batch=5000), dict(width=0), dict(n_pages=0), dict(page_size=0), dict(page_size=12),
    dict(page_size=1 << 20, width=1 << 12), dict(max_batch=4096, width=1 << 20), dict(other=dict(width=9)),
    dict(other=dict(ring=2 * P)), dict(other=dict(page_size=32)), dict(other=dict(max_batch=5)), dict(other=dict(table=None)),
    dict(rows=dict(slots=None)), dict(rows=dict(slots=P + 4)), dict(rows=dict(max_rows=0)), dict(rows=dict(granted=None)),
    dict(ctx=P + 2)])
def test_plan_refuses(lib, kw):
    assert _plan(lib, **kw) == EINVAL


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="CUDA"):
        paged.PageTables(torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        paged.PageRows(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        paged.PagedCache(torch.zeros(1, 2, 2, 16, 64), torch.zeros(1, 2, 2, 16, 64), 2)


def test_plan_model_on_a_hand_worked_step():
    m = TablesModel(n_pages=5, page=8, max_batch=3, width=4)
    r = m.plan([0, 0, 0], [9, 8, 20], 64)   # 2 + 1 pages; 3 more do not fit the 2 left
    assert m.tables == [[0, 1], [2], []] and (m.head, m.count) == (3, 2)
    assert r["row_start"] == [0, 9, 17, 37] and r["granted"] == [1, 1, 0] and r["seq_len"] == [9, 8, 0]
    assert r["slots"][:10] == [0, 1, 2, 3, 4, 5, 6, 7, 8, 16] and r["slots"][17] == -1
    r = m.plan([0, 8, 0], [0, 1, 0], 64)    # the first ends, the second goes on
    assert m.tables == [[], [2, 3], []] and (m.head, m.count) == (4, 3)
    assert [m.ring[(m.head + i) % 5] for i in range(3)] == [4, 0, 1]
    assert r["slots"][0] == 24 and r["positions"][0] == 8
