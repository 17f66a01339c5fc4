"""The paged key/value cache on the GPU against its definitions in fp64 (plan:
against a model on Python lists): types, head layouts, page sizes and orders, lengths
0, 1 and around tile edges, windows, masks that leave a row nothing, pages of NaN
around every request, refusals, streams and graphs."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged
from tests.paged_util import DTYPES, ROUND, Step, TablesModel, pack_mask

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- plan ------------------------------------------------------------------------------


def _same(tables, rows, model, r, b):
    width = model.width
    want = [t + [-1] * (width - len(t)) for t in model.tables]
    assert tables.table.tolist() == want
    assert tables.held.tolist() == [len(t) for t in model.tables]
    assert tables.state.tolist() == [model.head, model.count, 0, 0]
    n, ring = model.n_pages, tables.ring.tolist()
    assert [ring[(model.head + i) % n] for i in range(model.count)] == [model.ring[(model.head + i) % n] for i in range(model.count)]
    assert rows.row_start[:b + 1].tolist() == r["row_start"]
    for k in ("seq_len", "granted"):
        assert getattr(rows, k)[:b].tolist() == r[k], k
    assert rows.slots.tolist() == r["slots"]
    assert rows.positions.tolist() == r["positions"]


@pytest.mark.parametrize("batch,page,width,n_pages,max_rows,in_place", [
    (1, 16, 4, 6, 20, True), (7, 8, 9, 40, 150, True), (7, 8, 9, 40, 150, False), (33, 32, 5, 90, 700, True),
    (600, 16, 12, 3000, 9000, True), (1500, 64, 3, 2200, 30000, False)])
def test_plan_follows_the_model_over_many_steps(batch, page, width, n_pages, max_rows, in_place):
    rng = np.random.default_rng(batch + page)
    model = TablesModel(n_pages, page, batch, width)
    tables = paged.PageTables.empty(n_pages, page, batch, width)
    rows = paged.PageRows.empty(batch, max_rows)
    ctx = np.zeros(batch, np.int64)
    for step in range(12):
        b = batch if step % 3 else rng.integers(0, batch + 1)
        new = rng.integers(0, 2 * page, size=batch) * (rng.random(batch) < 0.7)
        ended = rng.random(batch) < 0.15
        ctx[ended], new[ended] = 0, 0
        if step == 5:
            new[0], ctx[-1] = -3, -1
        if step == 6:
            new[batch // 2] = width * page + 1
        if step == 7:
            ctx[0], new[0] = 2 ** 31 - 1, 2 ** 31 - 1
        c, n = ctx[:b].tolist(), new[:b].tolist()
        r = model.plan(c, n, max_rows)
        out = tables
        if not in_place:
            out = paged.PageTables(torch.full_like(tables.table, 7), torch.full_like(tables.held, 7), tables.ring,
                                   torch.zeros_like(tables.state), page)
            out.table[b:] = tables.table[b:]
            out.held[b:] = tables.held[b:]
            before = [t.clone() for t in (tables.table, tables.held, tables.state)]
        paged.plan(tables, rows, _i32(c), _i32(n), out=out)
        if not in_place:
            assert all(torch.equal(x, y) for x, y in zip(before, (tables.table, tables.held, tables.state)))
            tables = out
        _same(tables, rows, model, r, b)
        for i in range(batch):  # what was granted is committed in part, as a Jacobi step does
            if i < b and r["granted"][i]:
                ctx[i] += rng.integers(0, new[i] + 1)
            ctx[i] = min(max(int(ctx[i]), 0), width * page)
            if ctx[i] > len(model.tables[i]) * page:
                ctx[i] = len(model.tables[i]) * page


def test_plan_may_write_lengths_over_its_input():
    tables, rows = paged.PageTables.empty(40, 8, 4, 8), paged.PageRows.empty(4, 64)
    model = TablesModel(40, 8, 4, 8)
    rows.seq_len.copy_(_i32([5, 0, 9, 1]))
    paged.plan(tables, rows, rows.seq_len, _i32([3, 7, 0, 20]))
    _same(tables, rows, model, model.plan([5, 0, 9, 1], [3, 7, 0, 20], 64), 4)


def test_plan_refuses_mismatched_arguments():
    tables, rows = paged.PageTables.empty(40, 8, 4, 8), paged.PageRows.empty(4, 64)
    with pytest.raises(cllm.CllmError):
        paged.plan(tables, rows, _i32([0] * 4), _i32([1] * 4), out=paged.PageTables.empty(40, 8, 4, 8))  # another ring
    with pytest.raises(ValueError):
        paged.plan(tables, rows, _i32([0] * 5), _i32([1] * 5))
    with pytest.raises(ValueError):
        paged.plan(tables, rows, _i32([0] * 4), _i32([1] * 3))
    with pytest.raises(ValueError):
        paged.plan(tables, rows, torch.zeros(4, device="cuda"), _i32([1] * 4))


# ---- append ----------------------------------------------------------------------------


def _rope(max_pos, hd):
    i = torch.arange(hd // 2, dtype=torch.float64, device="cuda")
    ang = torch.arange(max_pos, dtype=torch.float64, device="cuda")[:, None] * 1e4 ** (-2 * i / hd)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


def _turned(x, rope, pos):
    cs = rope.double()[pos.long()][:, None]
    a, b = x.double().chunk(2, -1)
    out = torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)
    big = torch.cat([a.abs() + b.abs()] * 2, -1)
    return out, big


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,heads,kv,hd,page,order,rope", [
    (1, 4, 4, 64, 8, "page", True), (37, 12, 4, 128, 16, "token", True), (37, 4, 1, 64, 256, "page", True),
    (400, 5, 5, 128, 32, "page", True), (65, 28, 4, 128, 64, "token", False)])
def test_append(dtype, rows, heads, kv, hd, page, order, rope):
    dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(rows)
    rng = np.random.default_rng(rows)
    layers, n_pages = 3, 3 + 2 * -(-rows // page)
    shape = (layers, n_pages, kv, page, hd) if order == "page" else (layers, n_pages, page, kv, hd)
    kp, vp = (torch.randn(shape, device="cuda", generator=gen).to(dt) for _ in range(2))
    if order == "token":
        kp, vp = kp.transpose(2, 3), vp.transpose(2, 3)
    qkv = torch.randn(rows, (heads + 2 * kv) * hd, device="cuda", generator=gen).to(dt)
    q, k, v = (x.unflatten(1, (-1, hd)) for x in qkv.split([heads * hd, kv * hd, kv * hd], 1))
    slots = rng.permutation(n_pages * page)[:rows]
    slots[rng.random(rows) < 0.2] = -1
    slots = torch.from_numpy(slots).to("cuda")
    pos = torch.from_numpy(rng.integers(0, 500, rows).astype(np.int32)).to("cuda")
    table = _rope(500, hd)
    want_k, want_v = kp.double().clone(), vp.double().clone()
    u, live = ROUND[dtype], slots >= 0
    kk, kb = (_turned(k, table, pos) if rope else (k.double(), k.double().abs() * 0))
    pg, off = slots[live] // page, slots[live] % page
    want_k[1].transpose(1, 2)[pg, off] = kk[live]
    want_v[1].transpose(1, 2)[pg, off] = v.double()[live]
    tol = torch.zeros_like(want_k)
    # two products and a sum in fp32, then one rounding (none without rotation)
    tol[1].transpose(1, 2)[pg, off] = (3 * 2.0 ** -24 * kb + u * kk.abs() * (1 if rope else 0))[live]
    cache = paged.PagedCache(kp, vp, heads)
    if rope:
        qq, qb = _turned(q, table, pos)
        cache.append(1, k, v, slots, q=q, rope=table, positions=pos)  # in place
        assert bool(((q.double() - qq).abs() <= 3 * 2.0 ** -24 * qb + u * qq.abs() + 1e-30).all())
    else:
        before = qkv.clone()
        cache.append(1, k, v, slots)
        assert torch.equal(qkv, before)
    cache.check()
    assert bool(((kp.double() - want_k).abs() <= tol).all())
    assert torch.equal(vp.double(), want_v)


def test_append_skips_and_reports_what_is_outside():
    kp, vp = (torch.zeros(1, 4, 2, 8, 64, device="cuda", dtype=torch.float16) for _ in range(2))
    cache = paged.PagedCache(kp, vp, 2)
    k = torch.ones(4, 2, 64, device="cuda", dtype=torch.float16)
    slots = torch.tensor([3, 32, -5, 31], device="cuda")
    cache.append(0, k, k, slots)
    with pytest.raises(cllm.CllmError) as e:
        cache.check()
    assert e.value.status == -6
    cache.check()  # reported once
    for pool in (kp, vp):
        flat = pool[0].transpose(1, 2).reshape(32, -1).sum(1)
        assert flat.nonzero().flatten().tolist() == [3, 31]
    cache.append(0, k, k, torch.tensor([0, 1, 2, 4], device="cuda"), rope=_rope(10, 64), positions=_i32([0, 10, -1, 9]))
    with pytest.raises(cllm.CllmError):
        cache.check()
    assert kp[0].transpose(1, 2).reshape(32, -1).abs().sum(1).nonzero().flatten().tolist() == [0, 3, 4, 31]
    cache.append(0, k[:0], k[:0], slots)  # no rows: nothing to do
    cache.check()


def test_append_refusals():
    kp, vp = (torch.zeros(1, 4, 2, 8, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache = paged.PagedCache(kp, vp, 4)
    k = torch.zeros(3, 2, 64, device="cuda", dtype=torch.bfloat16)
    slots = torch.zeros(3, device="cuda", dtype=torch.int64)
    for bad in (dict(k=k.float()), dict(k=k[:, :1]), dict(k=k.cpu()), dict(slots=slots[:2]), dict(slots=slots.int()),
                dict(v=k[:2]), dict(q=torch.zeros(3, 4, 64, device="cuda", dtype=torch.bfloat16)),
                dict(rope=_rope(4, 128), positions=_i32([0] * 3)), dict(rope=_rope(4, 64), positions=_i32([0] * 2))):
        with pytest.raises(ValueError):
            cache.append(**{**dict(layer=0, k=k, v=k, slots=slots), **bad})
    with pytest.raises(cllm.CllmError):
        cache.append(1, k, k, slots)
    wide = torch.zeros(3 * 2 * 64 + 8, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(cllm.CllmError):  # rows that start off a 16-byte boundary
        cache.append(0, wide[1:385].view(3, 2, 64), k, slots)


# ---- attention -------------------------------------------------------------------------


def _check(step, mask=None, window=0, scale=None, out=None, q=None, tables=None, seq_len=None, far=None):
    cache = paged.PagedCache(step.k, step.v, step.heads)
    rows = paged.PageRows(step.row_start, step.seq_len if seq_len is None else _i32(seq_len))
    tables = tables or paged.PageTables(step.table, page_size=step.page)
    lse = torch.full((step.rows, step.heads), 7.0, device="cuda")
    bits = None if mask is None else pack_mask(mask)
    q = step.q if q is None else q
    got = cache.attention(step.layer, q, rows, tables, out=out, lse=lse, scale=scale, window=window, block_mask=bits)
    again = cache.attention(step.layer, q, rows, tables, scale=scale, window=window, block_mask=bits)
    cache.check()
    assert torch.equal(got, again)  # bit for bit
    o, want_lse, ab, delta = step.attention(scale, window, mask, seq_len)
    tol, ltol = step.bound(ab, delta, o)
    none = torch.isinf(want_lse)
    assert torch.equal(none, torch.isinf(lse))
    assert bool((got[none] == 0).all())
    err = (got.double() - o).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    lerr = (lse.double() - want_lse).abs()[~none]
    assert bool((lerr <= ltol[~none]).all()), float((lerr / ltol[~none]).max())
    return got


# requests around every edge: none, one and many cached tokens; none, one and many new ones
RAGGED = ([0, 1, 7, 127, 128, 129, 300, 64, 0, 513], [1, 1, 0, 1, 2, 7, 17, 33, 5, 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv,hd,page,order", [
    (4, 4, 64, 16, "page"), (4, 4, 128, 8, "token"), (8, 2, 128, 32, "page"), (7, 1, 64, 64, "token"),
    (12, 4, 128, 128, "page"), (64, 1, 64, 256, "page"), (5, 5, 128, 256, "token")])
def test_attention_ragged(dtype, heads, kv, hd, page, order):
    _check(Step(*RAGGED, heads, kv, hd, page, dtype, order, seed=heads + page, layers=2))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv,hd,page", [(4, 4, 128, 16), (6, 2, 64, 64), (7, 1, 128, 8)])
@pytest.mark.parametrize("ctx,new", [([0], [300]), ([257, 5], [128, 129]), ([100, 0, 40], [256, 257, 385])])
def test_attention_chunks(dtype, heads, kv, hd, page, ctx, new):
    _check(Step(ctx, new, heads, kv, hd, page, dtype, seed=sum(new)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 128, 200, 10000])
def test_attention_window(dtype, window):
    _check(Step(*RAGGED, 8, 2, 64, 16, dtype, seed=window), window=window)
    _check(Step([0, 300], [280, 40], 2, 2, 128, 32, dtype, seed=window + 1), window=window)


def test_attention_does_not_read_pages_before_the_window():
    step = Step([700], [3], 4, 2, 64, 16, "f16", seed=5)
    step.table[0, :(700 - 100) // 16] = -1  # given back
    cache = paged.PagedCache(step.k, step.v, 4)
    got = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16), window=80)
    cache.check()
    whole = Step([700], [3], 4, 2, 64, 16, "f16", seed=5)
    o, _, ab, delta = whole.attention(window=80)
    assert bool(((got.double() - o).abs() <= whole.bound(ab, delta, o)[0]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("ctx,new", [([0, 130, 40, 1], [5, 61, 33, 1]), ([64, 3], [130, 300])])
def test_attention_mask(dtype, window, ctx, new):
    """A random mask among the new tokens, rows without any bit among it: with no
    cached tokens they see nothing."""
    step = Step(ctx, new, 8, 2, 64, 16, dtype, seed=sum(new) + window)
    gen = torch.Generator().manual_seed(1)
    mask = torch.rand(step.rows, max(new), generator=gen) < 0.3
    mask[::4] = False
    _check(step, mask=mask, window=window)


def test_attention_mask_shorter_than_the_block():
    """Tokens past the mask's words are seen by no row."""
    step = Step([10], [70], 2, 2, 64, 8, "f16", seed=3)
    mask = torch.ones(70, 70, dtype=torch.bool)
    mask[:, 64:] = False
    cache = paged.PagedCache(step.k, step.v, 2)
    got = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=8),
                          block_mask=pack_mask(mask[:, :64]))
    o, _, ab, delta = step.attention(mask=mask)
    assert bool(((got.double() - o).abs() <= step.bound(ab, delta, o)[0]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("new", [4, 150])
def test_what_a_row_does_not_see_never_reaches_it(dtype, bad, new):
    """The last new tokens' keys and values are not numbers: the rows before them
    are what they are without."""
    step = Step([90, 0], [new, new], 4, 2, 64, 16, dtype, seed=new)
    o, lse, ab, delta = step.attention()
    tol, _ = step.bound(ab, delta, o)
    for b in range(2):
        for i in range(new - 3, new):
            step.token(step.k, b, step.ctx[b] + i)[...] = bad
            step.token(step.v, b, step.ctx[b] + i)[...] = bad
    cache = paged.PagedCache(step.k, step.v, 4)
    got = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16))
    cache.check()
    clean = [b * new + i for b in range(2) for i in range(new - 3)]
    assert bool(((got.double() - o).abs()[clean] <= tol[clean]).all())
    if not bad == -math.inf:
        assert bool((~torch.isfinite(got[new - 1])).all())
    mask = torch.tril(torch.ones(new, new, dtype=torch.bool)).repeat(2, 1)
    mask[:, new - 3:] = False  # nobody sees them
    seen = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16),
                           block_mask=pack_mask(mask))
    assert bool(torch.isfinite(seen).all())
    assert bool(((seen.double() - o).abs()[clean] <= tol[clean]).all())


# 17 to 64 rows a key/value head on average and enough heads, or groups of more than 16: tiles
# in 4 or 2 bands; among them tiles without tokens or keys, of one row, and cut ones
BANDS = [(32, 8, 64, 16, *RAGGED), (32, 8, 128, 32, *RAGGED), (20, 1, 128, 8, [0, 5, 200, 3000], [1, 0, 2, 1]),
         (32, 1, 64, 64, [2900], [1]), (33, 1, 128, 16, [100, 700], [1, 1]), (8, 1, 128, 64, [0, 1000, 63], [8, 5, 11]),
         (16, 16, 64, 8, [0, 100, 130, 64, 31, 200], [17, 32, 31, 1, 40, 3])]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,hd,page,ctx,new", BANDS)
@pytest.mark.parametrize("window,masked", [(0, False), (40, False), (0, True), (20, True)])
def test_attention_bands(dtype, heads, kv, hd, page, ctx, new, window, masked):
    step = Step(ctx, new, heads, kv, hd, page, dtype, seed=heads + window)
    mask = None
    if masked:
        mask = torch.rand(step.rows, max(new), generator=torch.Generator().manual_seed(2)) < 0.3
        mask[::3] = False
    _check(step, mask=mask, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("heads,kv,new", [(40, 40, 20), (24, 1, 2)])
def test_bands_keep_out_what_is_not_seen(dtype, bad, heads, kv, new):
    step = Step([90, 0], [new, new], heads, kv, 64, 16, dtype, seed=new)
    o, _, ab, delta = step.attention()
    tol, _ = step.bound(ab, delta, o)
    for b in range(2):
        for pool in (step.k, step.v):
            step.token(pool, b, step.ctx[b] + new - 1)[...] = bad
    cache = paged.PagedCache(step.k, step.v, heads)
    got = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16))
    cache.check()
    clean = [b * new + i for b in range(2) for i in range(new - 1)]
    assert bool(((got.double() - o).abs()[clean] <= tol[clean]).all())
    assert bool((~torch.isfinite(got[new - 1])).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_refused_requests_are_zeros(dtype):
    """A request that a plan refused has rows and a length of 0."""
    step = Step([100, 60, 7], [3, 140, 5], 4, 2, 64, 16, dtype, seed=2)
    got = _check(step, seq_len=[103, 0, 12])
    assert bool((got[3:143] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_attention_strides(dtype):
    """Queries between keys and values of one product, outputs with the heads outside."""
    step = Step([50, 300], [9, 140], 6, 2, 128, 32, dtype, seed=1)
    qkv = torch.full((step.rows, 10, 128), math.nan, device="cuda", dtype=step.q.dtype)
    qkv[:, 2:8] = step.q
    out = torch.full((6, step.rows + 1, 128), 3.0, device="cuda", dtype=step.q.dtype)
    _check(step, q=qkv[:, 2:8], out=out.transpose(0, 1)[:step.rows])
    assert bool((out[:, step.rows] == 3.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_long_context_and_scale(dtype):
    """Work cut over many CTAs, one token and a block; sharp and flat scores."""
    for scale in (None, 1.0, 1e-6):
        _check(Step([20001, 9000], [1, 12], 4, 1, 128, 64, dtype, seed=4), scale=scale)


def test_attention_offsets_past_32_bits():
    """Pages whose elements lie past 2^31 (and bytes past 2^32)."""
    page_elems = 2 * 256 * 128
    n = (1 << 31) // page_elems + 40
    step = Step([700, 90], [5, 140], 4, 2, 128, 256, "f16", seed=6, n_pages=n)
    assert int(step.table.max()) * page_elems > 1 << 31
    _check(step)
    k = torch.randn(3, 2, 128, device="cuda", dtype=torch.float16)
    cache = paged.PagedCache(step.k, step.v, 4)
    slots = torch.tensor([(n - 1) * 256 + 255, (n - 2) * 256 + 17, (n - 1) * 256], device="cuda")
    cache.append(0, k, k, slots)
    cache.check()
    assert all(torch.equal(pool[0, int(s) // 256, :, int(s) % 256], k[i]) for i, s in enumerate(slots) for pool in (step.k, step.v))


def test_attention_reports_pages_outside_the_pool():
    step = Step([100], [2], 4, 4, 64, 16, "f16")
    step.table[0, 1] = step.n_pages
    cache = paged.PagedCache(step.k, step.v, 4)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    cache.attention(0, step.q, rows, tables)
    with pytest.raises(cllm.CllmError) as e:
        cache.check()
    assert e.value.status == -6
    # rows past the arrays, lengths past the table: nothing is written out of bounds
    out = torch.full_like(step.q, 5.0)
    cache.attention(0, step.q, paged.PageRows(_i32([0, 1000]), step.seq_len), tables, out=out)
    with pytest.raises(cllm.CllmError):
        cache.check()
    assert bool((out == 5.0).all())
    cache.attention(0, step.q, paged.PageRows(step.row_start, _i32([10 ** 9])), tables, out=out)
    with pytest.raises(cllm.CllmError):
        cache.check()
    assert bool((out == 0.0).all())


def test_attention_refusals():
    step = Step([20], [3], 4, 2, 64, 16, "f16")
    cache = paged.PagedCache(step.k, step.v, 4)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    for bad in (dict(q=step.q.float()), dict(q=step.q[:, :2]), dict(q=step.q.cpu()), dict(out=step.q[:2]),
                dict(lse=torch.zeros(3, 4, device="cuda", dtype=torch.float64)),
                dict(tables=paged.PageTables(step.table, page_size=32)),
                dict(block_mask=torch.zeros(2, 1, device="cuda", dtype=torch.int32))):
        with pytest.raises(ValueError):
            cache.attention(**{**dict(layer=0, q=step.q, rows=rows, tables=tables), **bad})
    for bad in (dict(layer=1), dict(layer=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=3e38), dict(window=-1)):
        with pytest.raises(cllm.CllmError):
            cache.attention(**{**dict(layer=0, q=step.q, rows=rows, tables=tables), **bad})
    flat = torch.zeros(3 * 4 * 64 + 8, device="cuda", dtype=torch.float16)
    with pytest.raises(cllm.CllmError):
        cache.attention(0, flat[4:772].view(3, 4, 64), rows, tables)
    assert cache.attention(0, step.q[:0], rows, tables).shape == (0, 4, 64)


def test_allocation_failure():
    lib = cllm.load()
    step = Step([20], [3], 4, 2, 64, 16, "f16")
    lib.cllm_test_fail_alloc(0)
    with pytest.raises(cllm.CllmError) as e:
        paged.PagedCache(step.k, step.v, 4)
    assert e.value.status == -2
    lib.cllm_test_fail_alloc(-1)
    paged.PagedCache(step.k, step.v, 4).close()


@pytest.mark.parametrize("chunk", [0, 2])
@pytest.mark.parametrize("new", [3, 200])
def test_a_wait_that_runs_out_is_reported(chunk, new):
    """The MMA issuer gives up in every piece of more than `chunk` chunks: the call
    ends, the status says so, and the cache goes on working."""
    lib = cllm.load()
    step = Step([60000], [new], 2, 2, 128, 256, "bf16", seed=9)  # pieces of 7 chunks or so
    cache = paged.PagedCache(step.k, step.v, 2)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=256)
    want = cache.attention(0, step.q, rows, tables)
    cache.check()
    lib.cllm_test_hold_paged.argtypes = [ctypes.c_void_p, ctypes.c_int]
    assert lib.cllm_test_hold_paged(cache._h, chunk) == 0
    cache.attention(0, step.q, rows, tables)
    with pytest.raises(cllm.CllmError) as e:
        cache.check()
    assert e.value.status == -5
    assert lib.cllm_test_hold_paged(cache._h, -1) == 0
    assert torch.equal(cache.attention(0, step.q, rows, tables), want)
    cache.check()
    assert lib.cllm_test_hold_paged(None, 0) == -1 and lib.cllm_test_hold_paged(cache._h, -2) == -1


def test_a_wait_that_runs_out_in_bands_is_reported():
    lib = cllm.load()
    step = Step([60000], [1], 24, 1, 128, 256, "bf16", seed=9)
    cache = paged.PagedCache(step.k, step.v, 24)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=256)
    want = cache.attention(0, step.q, rows, tables)
    cache.check()
    lib.cllm_test_hold_paged.argtypes = [ctypes.c_void_p, ctypes.c_int]
    assert lib.cllm_test_hold_paged(cache._h, 1) == 0
    cache.attention(0, step.q, rows, tables)
    with pytest.raises(cllm.CllmError) as e:
        cache.check()
    assert e.value.status == -5
    assert lib.cllm_test_hold_paged(cache._h, -1) == 0
    assert torch.equal(cache.attention(0, step.q, rows, tables), want)
    cache.check()


# ---- together --------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_step_follows_the_lengths_on_the_device(dtype):
    """plan, append and attention captured once on a side stream, replayed while
    requests grow, end and start."""
    heads, kv, hd, page, batch, n = 4, 2, 64, 16, 3, 9
    dt = DTYPES[dtype]
    kp, vp = (torch.full((1, 40, kv, page, hd), math.nan, device="cuda", dtype=dt) for _ in range(2))
    cache = paged.PagedCache(kp, vp, heads)
    tables, rows = paged.PageTables.empty(40, page, batch, 10), paged.PageRows.empty(batch, batch * n)
    ctx, new = _i32([0] * batch), _i32([0] * batch)
    q, k, v = (torch.zeros(batch * n, h, hd, device="cuda", dtype=dt) for h in (heads, kv, kv))
    out, qr = torch.zeros_like(q), torch.zeros_like(q)
    rope = _rope(160, hd)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        paged.plan(tables, rows, ctx, new)
        cache.append(0, k, v, rows.slots, q=q, q_out=qr, rope=rope, positions=rows.positions)
        cache.attention(0, qr, rows, tables, out=out)
    gen = torch.Generator(device="cuda").manual_seed(0)
    kept = [[torch.zeros(0, kv, hd, device="cuda", dtype=torch.float64)] * 2 for _ in range(batch)]
    for step, lens in enumerate([[9, 0, 4], [1, 9, 9], [9, 9, 0], [0, 2, 9], [5, 9, 1]]):
        if step == 3:
            kept[1] = [x[:0] for x in kept[1]]  # a new request in place of the second
        ctx.copy_(_i32([c[0].shape[0] for c in kept]))
        new.copy_(_i32(lens))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        r = 0
        for b, m in enumerate(lens):
            pos = torch.arange(kept[b][0].shape[0], kept[b][0].shape[0] + m, device="cuda")
            ks = _turned(k[r:r + m], rope, pos)[0].to(dt).double()
            kept[b] = [torch.cat([kept[b][0], ks]), torch.cat([kept[b][1], v[r:r + m].double()])]
            kk, vv = (x.repeat_interleave(heads // kv, 1) for x in kept[b])
            qq = _turned(q[r:r + m], rope, pos)[0].to(dt).double()
            s = torch.einsum("ihd,khd->hik", qq, kk) * hd ** -0.5
            see = torch.arange(kk.shape[0], device="cuda")[None, :] <= pos[:, None]
            want = torch.einsum("hik,khd->ihd", s.masked_fill(~see, -math.inf).softmax(-1), vv)
            # one rounding of q, k (2 u of a score of at most ~8), p and o
            assert bool(((out[r:r + m].double() - want).abs() <= 40 * ROUND[dtype] + 1e-5).all())
            r += m
    cache.check()
    assert int(tables.state[1]) == 40 - int(tables.held.sum())
