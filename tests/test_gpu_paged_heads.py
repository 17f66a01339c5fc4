"""Rotary tables, and the write of keys with norms per head and rotations of part of the head, in
halves and in neighbours, against their definitions in fp64."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged
from tests.paged_util import DTYPES, ROUND

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- rotary tables ------------------------------------------------------------------------


def _true_table(positions, freq, amplitude, first):
    pos = np.arange(first, first + positions).astype(np.longdouble)[:, None]
    ang = pos * np.array(freq, np.float64).astype(np.longdouble)
    return float(np.float32(amplitude)) * np.stack([np.cos(ang), np.sin(ang)], -1)


@pytest.mark.parametrize("positions,dims", [(1, 2), (1, 128), (7, 6), (1000, 64), (4097, 128), (129, 34), (50, 256), (333, 2)])
@pytest.mark.parametrize("first", [0, 1, 100000])
def test_table(positions, dims, first):
    """In each value: 2^-22 of the amplitude, of which the table's own rounding is 2^-24."""
    f = paged.rope_frequencies(dims, 1e4)
    for amplitude in (1.0, 1.25):
        got = paged.rope_table(positions, f, amplitude, first)
        assert got.shape == (positions, dims // 2, 2)
        err = np.abs(got.cpu().numpy().astype(np.longdouble) - _true_table(positions, f, amplitude, first))
        assert float(err.max()) <= amplitude * 2.0 ** -22


def test_table_at_the_last_positions():
    """2^31 - 1 positions of any frequency: in 64-bit integers and fractions."""
    from fractions import Fraction
    pi = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)
    first, n = 2 ** 31 - 1 - 5, 5
    f = [1.0, 0.37, 1e-5, -0.2, 1000.1, 2.0 ** 20]
    got = paged.rope_table(n, f, first=first).double().cpu()
    for p in range(n):
        for i, x in enumerate(f):
            turn = Fraction(x) * (first + p) / (2 * pi)
            a = 2 * math.pi * float(turn - (turn.numerator // turn.denominator))
            assert abs(float(got[p, i, 0]) - math.cos(a)) <= 2.0 ** -22
            assert abs(float(got[p, i, 1]) - math.sin(a)) <= 2.0 ** -22


def test_table_rows_are_the_same_wherever_they_begin():
    f = paged.rope_frequencies(48, 5e5, "ramp", 8.0, trained=4096)
    whole = paged.rope_table(5000, f)
    out = torch.full((5002, 24, 2), 9.0, device="cuda")
    assert paged.rope_table(1234, f, first=3000, out=out[1:1235].view(1234, 24, 2)).data_ptr() == out[1].data_ptr()
    assert torch.equal(out[1:1235], whole[3000:4234])
    assert bool((out[0] == 9.0).all()) and bool((out[1235:] == 9.0).all())


def test_table_on_a_stream_and_in_a_graph():
    f = paged.rope_frequencies(64)
    want = paged.rope_table(300, f)
    side = torch.cuda.Stream()
    got = paged.rope_table(300, f, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        paged.rope_table(300, f, out=out)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_table_of_no_positions():
    assert paged.rope_table(0, [1.0, 0.5], first=7).shape == (0, 2, 2)


def test_table_refusals():
    out = torch.zeros(4, 2, 2, device="cuda")
    for kw in (dict(out=out.double()), dict(out=out[:3]), dict(out=out.transpose(0, 1)), dict(out=out.view(-1))):
        with pytest.raises(ValueError):
            paged.rope_table(4, [1.0, 0.5], **kw)
    for a in ((4, [1.0, math.nan]), (4, [0.5] * 129), (4, [0.5, 2.0 ** 21])):
        with pytest.raises(cllm.CllmError):
            paged.rope_table(*a)


# ---- writes ---------------------------------------------------------------------------------


def _normed(x, gain, eps):
    x = x.double()
    return x if gain is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()


def _turned(x, rope, pos, interleaved):
    """The rotated heads, and for every value the size of what it was made of."""
    if rope is None:
        return x, x.abs()
    cs, r = rope.double()[pos.long()][:, None], 2 * rope.shape[1]
    one, two = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b, y = x[..., one], x[..., two], x.clone()
    y[..., one], y[..., two] = a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]
    big = x.abs()
    big[..., one], big[..., two] = [(a.abs() + b.abs()) for _ in range(2)]
    return y, big


def _close(got, want, big, dtype, normed):
    """A norm: 20 roundings of the sum (half of them after the root), the root's reciprocal 4, four more
    products and sums: 24 of the value; a rotation two products and a sum; then one rounding, in fp16
    of values below 2^-14 (a rotation's sum may be any) to a multiple of 2^-24: off by up to 2^-25.  What
    is neither is a copy."""
    tol = (27 if normed else 3) * U32 * big + ROUND[dtype] * want.abs() + (2.0 ** -25 if dtype == "f16" else 1e-30)
    err = (got.double() - want).abs()
    worst = float((err / tol).max()) if err.numel() else 0.0
    assert worst <= 1.0, worst


CASES = [(1, 4, 4, 64, 8, "page"), (37, 12, 4, 128, 16, "token"), (19, 4, 1, 64, 256, "page"), (400, 5, 5, 128, 32, "page"),
         (3, 28, 4, 128, 64, "token"), (330, 64, 1, 64, 16, "token")]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,heads,kv,hd,page,order", CASES)
@pytest.mark.parametrize("dims,interleaved,norms", [(1.0, False, "qk"), (1.0, True, "qk"), (0.5, False, ""), (0.5, True, "k"),
                                                    (0.25, False, "q"), (0.75, False, "qk"), (0.25, True, ""), (1.0, True, ""),
                                                    (0, False, "qk"), (0, False, "k"), (0, False, "q")])
def test_append_heads(dtype, rows, heads, kv, hd, page, order, dims, interleaved, norms):
    dt, r = DTYPES[dtype], int(dims * hd)
    gen = torch.Generator(device="cuda").manual_seed(rows + r)
    rng = np.random.default_rng(rows + r)
    n_pages = 3 + 2 * -(-rows // page)
    shape = (2, n_pages, kv, page, hd) if order == "page" else (2, n_pages, page, kv, hd)
    kp, vp = (torch.randn(shape, device="cuda", generator=gen).to(dt) for _ in range(2))
    if order == "token":
        kp, vp = kp.transpose(2, 3), vp.transpose(2, 3)
    qkv = (3.0 * torch.randn(rows, (heads + 2 * kv) * hd, device="cuda", generator=gen)).to(dt)
    q, k, v = (x.unflatten(1, (-1, hd)) for x in qkv.split([heads * hd, kv * hd, kv * hd], 1))
    k[0, 0] = 0.0  # (its norm is eps alone)
    slots = rng.permutation(n_pages * page)[:rows]
    slots[rng.random(rows) < 0.2] = -1
    slots = torch.from_numpy(slots).to("cuda")
    rope = pos = None
    if r:
        rope = paged.rope_table(500, paged.rope_frequencies(r, 1e4))
        pos = torch.from_numpy(rng.integers(0, 500, rows).astype(np.int32)).to("cuda")
    gq, gk = ((1.0 + 0.5 * torch.randn(hd, device="cuda", generator=gen)).to(dt) if n in norms else None for n in "qk")
    eps = 1e-5
    want_q, big_q = _turned(_normed(q, gq, eps), rope, pos, interleaved)
    want_k, big_k = _turned(_normed(k, gk, eps), rope, pos, interleaved)
    before_k, before_v, before = kp.clone(), vp.clone(), qkv.clone()
    cache = paged.PagedCache(kp, vp, heads)
    q_out = torch.full((rows, heads, hd), 5.0, device="cuda", dtype=dt)
    kw = dict(rope=rope, positions=pos, q_norm=gq, k_norm=gk, eps=eps, interleaved=interleaved)
    cache.append(1, k, v, slots, q=q, q_out=q_out, **kw)
    cache.check()
    assert torch.equal(qkv, before)
    if not gq is None or r:
        _close(q_out, want_q, big_q, dtype, gq is not None)
    else:
        assert torch.equal(q_out, q)
    live = slots >= 0
    pg, off = slots[live] // page, slots[live] % page
    got_k, got_v = (p[1].transpose(1, 2)[pg, off] for p in (kp, vp))
    _close(got_k, want_k[live], big_k[live], dtype, gk is not None)
    assert torch.equal(got_v, v[live])
    for pool, old in ((kp, before_k), (vp, before_v)):  # nothing else is written
        pool[1].transpose(1, 2)[pg, off] = old[1].transpose(1, 2)[pg, off]
        assert torch.equal(pool, old)
    # in place, and without queries: the same
    cache.append(1, k, v, slots, q=q, **kw)
    assert torch.equal(q, q_out)
    if gq is None:
        again = kp[1].transpose(1, 2)[pg, off].clone()
        cache.append(1, k, v, slots, **kw)
        assert torch.equal(kp[1].transpose(1, 2)[pg, off], again)
    cache.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_whole_heads_in_halves_are_what_the_plain_call_writes(dtype):
    dt = DTYPES[dtype]
    k, q = (torch.randn(9, 4, 64, device="cuda").to(dt) for _ in range(2))
    slots, pos, rope = torch.arange(9, device="cuda"), _i32(list(range(9))), paged.rope_table(9, paged.rope_frequencies(64))
    pools = [torch.zeros(1, 2, 4, 8, 64, device="cuda", dtype=dt) for _ in range(4)]
    a, b = paged.PagedCache(pools[0], pools[1], 4), paged.PagedCache(pools[2], pools[3], 4)
    oa, ob = torch.empty_like(q), torch.empty_like(q)
    a.append(0, k, k, slots, q=q, q_out=oa, rope=rope, positions=pos)
    lib = paged.load()
    paged._ROWS_IN.pack_into(b._args, 0, 0, 9, k.data_ptr(), k.data_ptr(), q.data_ptr(), ob.data_ptr(), 256, 256, 256, 256,
                             slots.data_ptr(), rope.data_ptr(), pos.data_ptr(), 9)
    paged._HEADS.pack_into(b._args, paged._HEADS_AT, 0, 0, -1.0, 64, 0)
    assert lib.cllm_paged_append_heads(b._h, b._argp, b._argp + paged._HEADS_AT, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(oa, ob) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])


def test_append_heads_skips_rows_outside_the_table():
    kp, vp = (torch.zeros(1, 4, 2, 8, 64, device="cuda", dtype=torch.float16) for _ in range(2))
    cache = paged.PagedCache(kp, vp, 2)
    k, gain = torch.ones(4, 2, 64, device="cuda", dtype=torch.float16), torch.ones(64, device="cuda", dtype=torch.float16)
    cache.append(0, k, k, torch.tensor([0, 1, 32, 4], device="cuda"), rope=paged.rope_table(10, paged.rope_frequencies(32)),
                 positions=_i32([0, 10, 3, 9]), k_norm=gain, interleaved=True)
    with pytest.raises(cllm.CllmError) as e:
        cache.check()
    assert e.value.status == -6
    assert kp[0].transpose(1, 2).reshape(32, -1).abs().sum(1).nonzero().flatten().tolist() == [0, 4]


def test_append_heads_refusals():
    bf = dict(device="cuda", dtype=torch.bfloat16)
    kp, vp = (torch.zeros(1, 4, 2, 8, 64, **bf) for _ in range(2))
    cache = paged.PagedCache(kp, vp, 4)
    k, q, slots, gain = torch.zeros(3, 2, 64, **bf), torch.zeros(3, 4, 64, **bf), torch.zeros(3, device="cuda", dtype=torch.int64), torch.ones(64, **bf)
    pos = _i32([0] * 3)

    def table(pairs):
        return torch.zeros(4, pairs, 2, device="cuda")

    for bad in (dict(q_norm=gain), dict(q=q, q_norm=gain.float()), dict(q=q, q_norm=gain[:32]), dict(k_norm=gain.cpu()),
                dict(k_norm=torch.ones(128, **bf)[::2]),
                dict(rope=table(0), positions=pos), dict(rope=table(40), positions=pos), dict(rope=table(32)[..., 0], positions=pos),
                dict(rope=table(8)), dict(k_norm=gain, q=q[:2])):
        with pytest.raises(ValueError):
            cache.append(0, k, k, slots, **bad)
    for bad, status in ((dict(rope=table(4), positions=pos), -8), (dict(rope=table(20), positions=pos, interleaved=True), -8),
                        (dict(k_norm=gain, eps=-1.0), -1), (dict(k_norm=gain, eps=math.nan), -1), (dict(k_norm=gain, eps=math.inf), -1),
                        (dict(k_norm=torch.ones(65, **bf)[1:]), -1)):
        with pytest.raises(cllm.CllmError) as e:
            cache.append(0, k, k, slots, **bad)
        assert e.value.status == status
    assert not bool(kp.any()) and not bool(vp.any())
    cache.check()


def test_append_heads_replays_with_other_rows():
    dt = torch.bfloat16
    kp, vp = (torch.zeros(1, 6, 2, 8, 128, device="cuda", dtype=dt) for _ in range(2))
    cache = paged.PagedCache(kp, vp, 4)
    k, q, gain = torch.randn(5, 2, 128, device="cuda").to(dt), torch.randn(5, 4, 128, device="cuda").to(dt), torch.randn(128, device="cuda").to(dt)
    slots, pos, rope = torch.tensor([3, 4, 5, 6, 7], device="cuda"), _i32([3, 4, 5, 6, 7]), paged.rope_table(50, paged.rope_frequencies(64))
    out = torch.empty_like(q)
    kw = dict(q=q, q_out=out, rope=rope, positions=pos, q_norm=gain, k_norm=gain, interleaved=True)
    g = torch.cuda.CUDAGraph()
    cache.append(0, k, k, slots, **kw)
    with torch.cuda.graph(g):
        cache.append(0, k, k, slots, **kw)
    k.copy_(torch.randn(5, 2, 128, device="cuda"))
    slots.copy_(torch.tensor([40, -1, 12, 0, 47], device="cuda"))
    pos.copy_(_i32([40, 1, 12, 0, 47]))
    kp.zero_()
    g.replay()
    got, got_q = kp.clone(), out.clone()
    kp.zero_()
    cache.append(0, k, k, slots, **kw)
    assert torch.equal(kp, got) and torch.equal(out, got_q)
    assert int(kp[0].transpose(1, 2).reshape(48, -1).abs().sum(1).count_nonzero()) == 4


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_arguments_are_taken_alike_in_c_and_in_python(dtype, monkeypatch):
    """The native look at a call's tensors and the one in Python: the same calls, bit for bit."""
    dt = DTYPES[dtype]
    assert paged.load() is not None
    gen = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn(6, 8 * 64, device="cuda", generator=gen).to(dt)
    q, k, v = (x.unflatten(1, (-1, 64)) for x in qkv.split([4 * 64, 2 * 64, 2 * 64], 1))
    gain, slots, pos = torch.randn(64, device="cuda", generator=gen).to(dt), torch.tensor([3, 9, -1, 0, 15, 7, 99], device="cuda"), _i32(list(range(7)))
    f = paged.rope_frequencies(32)
    rope, whole = paged.rope_table(9, f), paged.rope_table(9, paged.rope_frequencies(64))
    calls = [dict(), dict(rope=whole, positions=pos), dict(rope=whole, positions=pos, q=q), dict(rope=rope, positions=pos, q=q, interleaved=True),
             dict(k_norm=gain), dict(interleaved=True), dict(k_norm=gain, interleaved=True), dict(q=q, k_norm=gain), dict(q=q, q_norm=gain, k_norm=gain, eps=0.25, rope=rope, positions=pos)]
    for kw in calls:
        got = []
        for native in (True, False):
            pools = [torch.zeros(1, 2, 2, 8, 64, device="cuda", dtype=dt) for _ in range(2)]
            cache = paged.PagedCache(*pools, 4)
            if not native:
                monkeypatch.setattr(cache, "_append", None)
            out = torch.zeros(6, 4, 64, device="cuda", dtype=dt)
            cache.append(0, k, v, slots, **kw, **({"q_out": out} if "q" in kw else {}))
            cache.check()
            got.append([*pools, out])
        assert all(torch.equal(a, b) for a, b in zip(*got))
    if paged._marshal is not None:  # what is not taken there is refused in Python, as without it
        cache.close()
        with pytest.raises(cllm.CllmError):
            cache.append(0, k, v, slots)
        table = torch.zeros(9, 16, 2, device="cuda")
        assert paged.rope_table(9, list(f), out=table) is table and torch.equal(table, rope)
        monkeypatch.setattr(paged, "_marshal", None)
        assert torch.equal(paged.rope_table(9, f, out=torch.zeros_like(table)), rope)


def test_a_table_past_31_bits():
    """2^25 + 3 positions of 64 pairs: 2^31 pairs and more."""
    n, f = 2 ** 25 + 3, paged.rope_frequencies(128, 1e6)
    got = paged.rope_table(n, f)
    for first in (0, 2 ** 24 - 2, n - 5):
        part = got[first:first + 5].cpu().numpy().astype(np.longdouble)
        assert float(np.abs(part - _true_table(5, f, 1.0, first)).max()) <= 2.0 ** -22
        assert torch.equal(got[first:first + 5], paged.rope_table(5, f, first=first))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_append_heads_past_31_bits(dtype):
    """Rows and pages whose values begin past 2^31."""
    dt, rows = DTYPES[dtype], 2 ** 22 + 3
    pools = [torch.zeros(1, 2 ** 13 + 2, 8, 256, 128, device="cuda", dtype=dt) for _ in range(2)]
    cache = paged.PagedCache(*pools, 8)
    slots = torch.full((rows,), -1, device="cuda")
    last = (2 ** 13 + 1) * 256 + 255
    slots[-2:] = torch.tensor([last, last - 300], device="cuda")
    pos, rope, gain = torch.zeros(rows, dtype=torch.int32, device="cuda"), paged.rope_table(9, paged.rope_frequencies(64)), torch.ones(128, device="cuda", dtype=dt)
    pos[-2:] = _i32([8, 3])
    q = torch.empty(rows, 8, 128, device="cuda", dtype=dt)
    q.normal_()
    before, out = q[-2:].clone(), torch.empty_like(q)
    cache.append(0, q, q, slots, q=q, q_out=out, rope=rope, positions=pos, q_norm=gain, k_norm=gain)  # (not in place: q is k)
    cache.check()
    small = [torch.zeros(1, 2, 8, 256, 128, device="cuda", dtype=dt) for _ in range(2)]
    other = paged.PagedCache(*small, 8)
    want = before.clone()
    other.append(0, before, before, torch.tensor([3, 4], device="cuda"), q=before, q_out=want, rope=rope, positions=_i32([8, 3]), q_norm=gain, k_norm=gain)
    assert torch.equal(out[-2:], want)
    for row, s in ((0, last), (1, last - 300)):
        assert torch.equal(pools[0][0, s // 256, :, s % 256], small[0][0, 0, :, 3 + row])
