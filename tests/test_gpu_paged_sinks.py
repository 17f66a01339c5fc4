"""Attention within a window beside which a request's first tokens stay visible, against its definition
in fp64: windows and first tokens around every edge of chunks, tiles and pages, masks, tiles of all
kinds, pages between that are gone or hold NaN."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged
from tests.paged_util import Step, pack_mask

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _definition(step, window, sinks, mask=None, lens=None, scale=None):
    """(out, lse, sum p |v|, largest score error's scale) in fp64, as Step.attention gives them."""
    scale = step.hd ** -0.5 if scale is None else scale
    dev, g = step.q.device, step.heads // step.kv_heads
    o = torch.zeros(step.rows, step.heads, step.hd, dtype=torch.float64, device=dev)
    ab, lse = torch.zeros_like(o), torch.full((step.rows, step.heads), -math.inf, dtype=torch.float64, device=dev)
    delta = torch.zeros_like(lse)
    lens, starts = step.seq_len.tolist() if lens is None else lens, step.row_start.tolist()
    for b, n in enumerate(step.new):
        ctx = lens[b] - n
        if n == 0 or ctx < 0:
            continue
        pos = torch.arange(lens[b], device=dev)
        at = step.table[b].long()[pos // step.page].clamp(min=0)
        k, v = (p[step.layer][at, :, pos % step.page].double() for p in (step.k, step.v))
        for i in range(n):
            r = starts[b] + i
            see = pos <= ctx + i if mask is None else torch.cat([torch.ones(ctx, dtype=torch.bool, device=dev), mask[r, :n].to(dev)])
            see = see & ((ctx + i - pos < window) | (pos < sinks))
            if not bool(see.any()):
                continue
            kk, vv = k[see].repeat_interleave(g, 1), v[see].repeat_interleave(g, 1)
            qr = step.q[r].double()
            s = torch.einsum("hd,khd->hk", qr, kk) * scale
            lse[r] = torch.logsumexp(s, -1)
            p = (s - lse[r][:, None]).exp()
            o[r], ab[r] = torch.einsum("hk,khd->hd", p, vv), torch.einsum("hk,khd->hd", p, vv.abs())
            delta[r] = (torch.einsum("hd,khd->hk", qr.abs(), kk.abs()) * scale).amax(-1)
    return o, lse, ab, delta


def _drop_pages(step, window, sinks):
    """Table entries of pages that no row of a request sees."""
    for b, n in enumerate(step.new):
        oldest = int(step.seq_len[b]) - n - window + 1
        first = -(-sinks // step.page)
        step.table[b, first:max(first, oldest // step.page)] = -1


def _check(step, window, sinks, mask=None, drop=True):
    want = _definition(step, window, sinks, mask)
    if drop:
        _drop_pages(step, window, sinks)
    cache = paged.PagedCache(step.k, step.v, step.heads)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=step.page)
    lse = torch.full((step.rows, step.heads), 7.0, device="cuda")
    bits = None if mask is None else pack_mask(mask)
    got = cache.attention(step.layer, step.q, rows, tables, lse=lse, window=window, block_mask=bits, sinks=sinks)
    again = cache.attention(step.layer, step.q, rows, tables, window=window, block_mask=bits, sinks=sinks)
    cache.check()
    assert torch.equal(got, again)  # bit for bit
    o, want_lse, ab, delta = want
    tol, ltol = step.bound(ab, delta, o)
    none = torch.isinf(want_lse)
    assert torch.equal(none, torch.isinf(lse))
    assert bool((got[none] == 0).all())
    worst = float(((got.double() - o).abs() / tol).max())
    assert worst <= 1.0, worst
    if not bool(none.all()):
        worst = float(((lse.double() - want_lse).abs() / ltol)[~none].max())
        assert worst <= 1.0, worst
    return got


# requests around every edge: none, one and many cached tokens; none, one and many new ones
RAGGED = ([0, 1, 7, 127, 128, 129, 300, 64, 0, 513], [1, 1, 0, 1, 2, 7, 17, 33, 5, 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv,hd,page,order", [
    (4, 4, 64, 16, "page"), (4, 4, 128, 8, "token"), (8, 2, 128, 32, "page"), (7, 1, 64, 64, "token"), (64, 1, 64, 256, "page")])
@pytest.mark.parametrize("window,sinks", [(1, 1), (20, 4), (64, 64), (5, 63), (100, 65), (200, 128), (3, 129), (50, 300), (1, 10000)])
def test_ragged(dtype, heads, kv, hd, page, order, window, sinks):
    _check(Step(*RAGGED, heads, kv, hd, page, dtype, order, seed=heads + sinks, layers=2), window, sinks)


CHUNKS = [([0], [300]), ([257, 5], [128, 129]), ([700, 40], [290, 257])]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv,hd,page", [(4, 4, 128, 16), (6, 2, 64, 64), (7, 1, 128, 8)])
@pytest.mark.parametrize("ctx,new", CHUNKS)
@pytest.mark.parametrize("window,sinks", [(30, 4), (129, 70), (64, 260), (500, 130)])
def test_chunks(dtype, heads, kv, hd, page, ctx, new, window, sinks):
    """Tiles of 64 and 128 rows, whose rows' windows begin in other chunks."""
    _check(Step(ctx, new, heads, kv, hd, page, dtype, seed=sum(new) + sinks), window, sinks)


@pytest.mark.parametrize("ctx,new,window,sinks", [(*CHUNKS[0], 30, 4), (*CHUNKS[0], 129, 70), (*CHUNKS[0], 64, 260), (*CHUNKS[0], 500, 130),
                                                  (*CHUNKS[1], 129, 70), (*CHUNKS[2], 129, 70), (*CHUNKS[2], 30, 4)])
def test_tiles_of_256_rows(ctx, new, window, sinks):
    """(80 heads: as many tiles as SMs.)  The second half's window begins after the first's, behind first tokens
    that both see."""
    _check(Step(ctx, new, 80, 80, 64, 32, "f16", seed=sum(new) + sinks), window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("new", [1, 5, 40, 200])
@pytest.mark.parametrize("window,sinks,page", [(2500, 4, 16), (2100, 700, 64), (1999, 129, 8)])
def test_long_windows_are_cut(dtype, new, window, sinks, page):
    """Tiles in parts: first tokens and window in other parts, and in one."""
    _check(Step([4000], [new], 4, 2, 128, page, dtype, seed=new), window, sinks)
    _check(Step([4000, 10, 2700], [new, 3, 1], 2, 1, 64, page, dtype, seed=new + 1), window, sinks)


BANDS = [(32, 8, 64, 16, *RAGGED), (20, 1, 128, 8, [0, 5, 200, 3000], [1, 0, 2, 1]), (32, 1, 64, 64, [2900], [1]),
         (8, 1, 128, 64, [0, 1000, 63], [8, 5, 11]), (16, 16, 64, 8, [0, 100, 130, 64, 31, 200], [17, 32, 31, 1, 40, 3])]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,hd,page,ctx,new", BANDS)
@pytest.mark.parametrize("window,sinks,masked", [(40, 4, False), (150, 100, False), (20, 33, True)])
def test_bands(dtype, heads, kv, hd, page, ctx, new, window, sinks, masked):
    step = Step(ctx, new, heads, kv, hd, page, dtype, seed=heads + window)
    mask = torch.rand(step.rows, max(new), generator=torch.Generator().manual_seed(2)) < 0.5 if masked else None
    _check(step, window, sinks, mask)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("window,sinks", [(20, 4), (3, 50), (70, 200)])
@pytest.mark.parametrize("ctx,new", [([0, 130, 40, 1], [5, 61, 33, 1]), ([64, 3, 0], [130, 300, 60])])
def test_mask(dtype, window, sinks, ctx, new):
    """A random mask among the new tokens, which first tokens may be; rows without any bit among it."""
    step = Step(ctx, new, 8, 2, 64, 16, dtype, seed=sum(new) + window)
    mask = torch.rand(step.rows, max(new), generator=torch.Generator().manual_seed(1)) < 0.3
    mask[::4] = False
    _check(step, window, sinks, mask)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("new", [2, 150])
def test_what_lies_between_never_reaches_a_row(dtype, bad, new):
    """Keys and values between the first tokens and the oldest window are not numbers, in pages that are
    read too; pages wholly between are gone."""
    window, sinks = 70, 5
    step = Step([400, 0, 90], [new, new, new], 4, 2, 64, 32, dtype, seed=new)
    o, lse, ab, delta = _definition(step, window, sinks)
    tol, _ = step.bound(ab, delta, o)
    for b in range(3):
        for pos in range(sinks, max(sinks, step.ctx[b] - window + 1)):
            step.token(step.k, b, pos)[...] = bad
            step.token(step.v, b, pos)[...] = bad
    _drop_pages(step, window, sinks)
    cache = paged.PagedCache(step.k, step.v, 4)
    got = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=32),
                          window=window, sinks=sinks)
    cache.check()
    assert bool(((got.double() - o).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_values_that_other_rows_see_never_reach_a_row(dtype):
    """The oldest row's window and later rows' values hold infinities; first tokens are all rows'."""
    window, sinks, new = 40, 6, 60
    step = Step([200], [new], 4, 2, 64, 16, dtype, seed=9)
    for pos in range(200 - 39, 200 - 20):  # row i sees from 161 + i on: the last of these, 179, up to row 18
        step.token(step.v, 0, pos)[...] = math.inf
    o, _, ab, delta = _definition(step, window, sinks)
    tol, _ = step.bound(ab, delta, o)
    cache = paged.PagedCache(step.k, step.v, 4)
    got = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16),
                          window=window, sinks=sinks)
    clean = list(range(19, new))
    assert bool(torch.isfinite(o[clean]).all())
    assert bool(((got.double() - o).abs()[clean] <= tol[clean]).all())
    assert not bool(torch.isfinite(got[:19]).any())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("new", [1, 100])
def test_without_a_window_first_tokens_change_nothing(dtype, new):
    step = Step([300, 20], [new, new], 4, 2, 64, 16, dtype, seed=new)
    cache = paged.PagedCache(step.k, step.v, 4)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    want = cache.attention(0, step.q, rows, tables)
    assert torch.equal(cache.attention(0, step.q, rows, tables, sinks=7), want)
    assert torch.equal(cache.attention(0, step.q, rows, tables, window=2 ** 31 - 1, sinks=2 ** 31 - 1), want)
    assert torch.equal(cache.attention(0, step.q, rows, tables, window=64, sinks=0),
                       cache.attention(0, step.q, rows, tables, window=64))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads", [4, 40])
def test_refused_requests_and_rows_behind_the_last(dtype, heads):
    step = Step([300, 50, 80], [3, 4, 2], heads, 1, 64, 16, dtype, seed=3)
    cache = paged.PagedCache(step.k, step.v, heads)
    rows = paged.PageRows(step.row_start, _i32([303, 0, 1]))  # the second refused, the third shorter than its rows
    q = torch.cat([step.q, step.q[:2]])
    out, lse = torch.full_like(q, 5.0), torch.full((11, heads), 5.0, device="cuda")
    cache.attention(0, q, rows, paged.PageTables(step.table, page_size=16), out=out, lse=lse, window=20, sinks=4)
    cache.check()
    o, _, ab, delta = _definition(step, 20, 4, lens=[303, 0, 1])
    assert bool(((out[:9].double() - o).abs() <= step.bound(ab, delta, o)[0]).all())
    assert bool((out[3:9] == 0).all()) and bool(torch.isinf(lse[3:9]).all())
    assert bool((out[9:] == 5.0).all()) and bool((lse[9:] == 5.0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads,new", [(2, 1), (40, 1), (2, 70)])
def test_the_longest_request(dtype, heads, new):
    """2^31 - 8192 tokens or a few less, of which some pages are left."""
    page, window, sinks = 256, 300, 130
    near = Step([700], [new], heads, 1, 64, page, dtype, seed=4)  # its first page stays, the others move to the end
    gap = (2 ** 31 - 8192 - 700 - new) // page * page
    total = 700 + new + gap
    table = torch.full((1, -(-total // page)), -1, dtype=torch.int32, device="cuda")
    used = -(-(700 + new) // page)
    table[0, 0] = near.table[0, 0]
    table[0, gap // page + 1:gap // page + used] = near.table[0, 1:used]
    cache = paged.PagedCache(near.k, near.v, heads)
    got = cache.attention(0, near.q, paged.PageRows(near.row_start, _i32([total])), paged.PageTables(table, page_size=page),
                          window=window, sinks=sinks)
    cache.check()
    o, _, ab, delta = _definition(near, window, sinks)
    assert bool(((got.double() - o).abs() <= near.bound(ab, delta, o)[0]).all())


def test_a_page_that_is_seen_and_gone_is_reported():
    for lost in (0, 15):
        step = Step([240], [2], 4, 2, 64, 16, "f16", seed=1)
        _drop_pages(step, 20, 4)
        step.table[0, lost] = -1
        cache = paged.PagedCache(step.k, step.v, 4)
        cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16),
                        window=20, sinks=4)
        with pytest.raises(cllm.CllmError) as e:
            cache.check()
        assert e.value.status == -6


def test_refusals():
    step = Step([20], [3], 4, 2, 64, 16, "f16")
    cache = paged.PagedCache(step.k, step.v, 4)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    out = torch.full_like(step.q, 5.0)
    for kw in (dict(sinks=-1, window=4), dict(sinks=-1), dict(sinks=4, window=-1)):
        with pytest.raises(cllm.CllmError):
            cache.attention(0, step.q, rows, tables, out=out, **kw)
    with pytest.raises(ValueError, match="sinks"):
        cache.attention(0, step.q, rows, tables, out=out, window=4, sinks=2 ** 32 + 4)
    assert bool((out == 5.0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_a_captured_step_replays_with_other_lengths(dtype):
    step = Step([400, 30], [4, 4], 4, 2, 64, 16, dtype, seed=6)
    cache = paged.PagedCache(step.k, step.v, 4)
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    out = torch.empty_like(step.q)
    kw = dict(out=out, window=50, sinks=9)
    cache.attention(0, step.q, rows, tables, **kw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attention(0, step.q, rows, tables, **kw)
    for lens in ([404, 34], [60, 4], [333, 20]):
        step.seq_len.copy_(_i32(lens))
        g.replay()
        got = out.clone()
        cache.attention(0, step.q, rows, tables, **kw)
        assert torch.equal(got, out)
        o, _, ab, delta = _definition(step, 50, 9, lens=lens)
        assert bool(((got.double() - o).abs() <= step.bound(ab, delta, o)[0]).all())
    cache.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_arguments_are_taken_alike_in_c_and_in_python(dtype, monkeypatch):
    """The native look at a call's tensors and the one in Python: the same results and refusals."""
    step = Step([300, 20], [5, 7], 4, 2, 64, 16, dtype, seed=8)
    wide = torch.zeros(12, 4, 96, device="cuda", dtype=step.q.dtype)
    wide[..., :64] = step.q
    rows, tables = paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16)
    mask = pack_mask(torch.rand(12, 7, generator=torch.Generator().manual_seed(3)) < 0.6)
    got = []
    for native in (True, False):
        cache = paged.PagedCache(step.k, step.v, 4)
        if not native:
            monkeypatch.setattr(cache, "_attention", None)
        results = []
        for kw in (dict(), dict(window=30, sinks=4), dict(window=30, sinks=4, block_mask=mask), dict(scale=0.3), dict(out=wide[..., 32:])):
            lse = torch.zeros(12, 4, device="cuda")
            q = step.q if "out" in kw else wide[..., :64]
            results += [cache.attention(0, q, rows, tables, lse=lse, **kw).clone(), lse]
        cache.check()
        got.append(results)
        wide[..., :64] = step.q
        for bad in (dict(lse=lse[:5]), dict(lse=lse.double()), dict(q=step.q[:, :3]), dict(q=step.q.cpu()), dict(out=step.q.double()),
                    dict(block_mask=mask[:5]), dict(block_mask=mask.long()), dict(tables=paged.PageTables(step.table, page_size=32))):
            with pytest.raises(ValueError):
                cache.attention(**{**dict(layer=0, q=step.q, rows=rows, tables=tables), **bad})
        for bad in (dict(layer=1), dict(window=-1), dict(scale=-1.0), dict(scale=math.nan), dict(out=step.q)):
            with pytest.raises(cllm.CllmError):
                cache.attention(**{**dict(layer=0, q=step.q, rows=rows, tables=tables), **bad})
    assert all(torch.equal(a, b) for a, b in zip(*got))
    cache.close()
    with pytest.raises(cllm.CllmError):
        cache.attention(0, step.q, rows, tables)
