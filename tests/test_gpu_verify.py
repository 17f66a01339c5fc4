"""Draft verification on the GPU against its definition in fp64: types, vocabularies of one to many
thousand and odd sizes, strides, requests of no and many rows, temperatures, logits that are no
numbers, ties, drafts that are none, streams, graphs; and the distribution of what it draws."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged, verify
from tests.paged_util import DTYPES
from tests.verify_util import TOL, Model

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Batch:
    """Requests of n rows each: logits with a favourite a row, drafts that name it often, random numbers."""

    def __init__(self, n, vocab, dtype="f32", probs=False, heat=None, seed=0, pad=0, offset=0, peak=2.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.n, self.vocab, self.t = n, vocab, sum(n)
        z = 2.0 * torch.randn(self.t, vocab, device="cuda", generator=g)
        best = torch.randint(0, vocab, (self.t,), device="cuda", generator=g)
        z[torch.arange(self.t, device="cuda"), best] = math.log(vocab) + peak
        room = torch.full((self.t * (vocab + pad) + offset,), float("nan"), device="cuda", dtype=DTYPES[dtype])
        self.z = room[offset:].view(self.t, vocab + pad)[:, :vocab]
        self.z.copy_(z)
        self.probs = torch.softmax(z + 0.5 * torch.randn(z.shape, device="cuda", generator=g), -1) if probs else None
        follow = best.clone()
        other = torch.from_numpy(rng.random(self.t) < 0.3).to("cuda")
        follow[other] = torch.randint(0, vocab, (int(other.sum()),), device="cuda", generator=g)
        if probs:
            follow = (self.probs / torch.empty_like(z).exponential_(generator=g)).argmax(-1)
        tokens = torch.randint(0, vocab, (self.t,), device="cuda", generator=g)
        tokens[1:] = follow[:-1]
        self.tokens = tokens.int()
        self.u = torch.rand(self.t, device="cuda", generator=g)
        self.race = torch.empty(len(n), vocab, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
        self.heat = None if heat is None else torch.tensor(heat, dtype=torch.float32, device="cuda")
        start = np.concatenate([[0], np.cumsum(n)])
        self.start = start
        self.rows = paged.PageRows(_i32(start.tolist()), _i32([x + 10 for x in n]))

    def call(self, verifier=None, **kw):
        v = verifier or verify.DraftVerifier(max(self.t, 1), len(self.n))
        p = torch.full((self.t,), 7.0, device="cuda")
        args = dict(uniforms=self.u, race=self.race, temperature=self.heat, draft_probs=self.probs, target_probs=p)
        a, x = v.verify(self.z, self.tokens, self.rows, **{**args, **kw})
        again = v.verify(self.z, self.tokens, self.rows, **{**args, **kw})
        assert torch.equal(a, again[0]) and torch.equal(x, again[1])
        return a.tolist(), x.tolist(), p.double().cpu().numpy()

    def models(self, greedy=False):
        z, u, race = self.z.double().cpu().numpy(), self.u.double().cpu().numpy(), self.race.double().cpu().numpy()
        tokens = self.tokens.tolist()
        heat = [1.0] * len(self.n) if self.heat is None else self.heat.tolist()
        q = None if self.probs is None else self.probs.cpu().numpy()
        for b, (r, n) in enumerate(zip(self.start, self.n)):
            s = slice(r, r + n)
            yield None if n == 0 else Model(z[s], tokens[s], None if greedy else race[b], u[s], heat[b], None if q is None or greedy else q[s])

    def check(self, greedy=False, **kw):
        if greedy:
            kw = dict(uniforms=None, race=None, temperature=None, draft_probs=None, **kw)
        accepted, following, p = self.call(**kw)
        for b, m in enumerate(self.models(greedy)):
            if m is None:
                assert (accepted[b], following[b]) == (0, -1)
                continue
            assert m.allows(accepted[b], following[b]), (b, accepted[b], following[b], m.accepted, m.next)
            got = p[self.start[b]:self.start[b] + self.n[b]]
            assert (np.abs(got - m.probs) <= 2 * TOL * m.probs + 2.0 ** -149).all()
        return accepted, following


RAGGED = [1, 5, 0, 16, 2, 0, 33, 3, 70]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 64, 255, 2048, 2049, 32001])
@pytest.mark.parametrize("probs", [False, True])
def test_ragged(dtype, vocab, probs):
    heat = [1.0, 0.0, 1.0, 0.7, 1.3, 0.0, 0.5, 0.0, 2.0]
    Batch(RAGGED, vocab, dtype, probs, None, seed=vocab).check()
    Batch(RAGGED, vocab, dtype, probs, heat, seed=vocab + 1).check()
    Batch(RAGGED, vocab, dtype, seed=vocab + 2).check(greedy=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,rows,vocab", [(1, 1, 50000), (1, 16, 32000), (3, 4, 131072), (200, 3, 4001), (700, 2, 300), (1, 500, 3001)])
def test_shares_of_rows_and_vocabularies(dtype, batch, rows, vocab):
    Batch([rows] * batch, vocab, dtype, batch < 4, seed=rows).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (16, 7)])
@pytest.mark.parametrize("vocab", [5, 4096, 5003])
def test_rows_that_begin_anywhere(dtype, pad, offset, vocab):
    """Logits between the rows are NaN; race and draft rows have strides of their own."""
    b = Batch([4, 9, 1], vocab, dtype, True, seed=pad + vocab, pad=pad, offset=offset)
    race = torch.full((3, vocab + 3), float("nan"), device="cuda")[:, 1:vocab + 1]
    race.copy_(b.race)
    probs = torch.full((b.t, vocab + 2), float("nan"), device="cuda")[:, 2:]
    probs.copy_(b.probs)
    want = b.check()
    assert b.call(race=race, draft_probs=probs)[:2] == want
    b.check(greedy=True)


def test_long_runs_of_drafts_that_stand():
    """Requests of 33 to 200 rows whose drafts all stand, or fall at a chosen row."""
    n = [33, 64, 65, 200, 100]
    b = Batch(n, 97, peak=60.0, seed=3)
    b.tokens[1:] = b.z.argmax(-1)[:-1].int()
    assert b.check()[0] == n
    for row, request in ((0, 0), (31, 1), (32, 2), (190, 3), (98, 4)):
        at = int(b.start[request]) + row
        b.tokens[at + 1] = (int(b.z[at].argmax()) + 1) % 97
    assert b.check()[0] == [1, 32, 33, 191, 99]
    assert b.check(greedy=True)[0] == [1, 32, 33, 191, 99]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_ties_go_to_the_lowest_index(dtype):
    vocab = 5003
    b = Batch([2, 2, 2], vocab, dtype, seed=1)
    b.z.zero_()
    b.z[0, [17, 4000, 4999]] = 3.0
    b.z[2, [0, 5002]] = 3.0
    b.z[4] = -2.0
    b.tokens.copy_(_i32([0, 4000, 0, 0, 0, 1]))
    assert b.check(greedy=True) == ([1, 2, 1], [17, 0, 0])
    b.z[2:4] = torch.tensor([0.0, -0.0], device="cuda").repeat(2, vocab)[:, :vocab].to(b.z.dtype)  # (equal too)
    assert b.check(greedy=True)[1][1] == 0
    b.race.fill_(1.0)
    b.u.fill_(0.999)
    assert b.check() == ([1, 1, 1], [17, 1, 0])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heat", [None, [0.0] * 4])
def test_rows_without_a_distribution(dtype, bad, heat):
    """-inf: all of a row (one is a token that is never drawn); the rows before decide if they can."""
    vocab = 4099
    b = Batch([6, 6, 3, 1], vocab, dtype, heat=heat, seed=2, peak=60.0 if dtype != "f16" else 30.0)
    b.tokens[1:] = b.z.argmax(-1)[:-1].int()
    rows = [3, 6 + 5, 12, 15]
    for r in rows:
        if bad == -math.inf:
            b.z[r] = bad
        else:
            b.z[r, (37 * r) % vocab] = bad
    accepted, following = b.check()
    if bad != math.inf or heat is None:
        assert accepted == [4, 6, 1, 1] and following == [-1] * 4
    b.check(greedy=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masked_logits_are_never_drawn(dtype):
    for seed in range(5):
        b = Batch([3] * 40, 1000, dtype, seed % 2 == 1, seed=seed)
        allowed = torch.rand(b.t, 1000, device="cuda") < 0.01
        allowed[:, 5] = True
        b.z.masked_fill_(~allowed, -math.inf)
        accepted, following = b.check()
        for r, a, x in zip(b.start, accepted, following):
            assert bool(allowed[r + a - 1, x])


def test_temperatures_at_and_past_their_ends():
    heat = [0.0, 2.0 ** -61, 2.0 ** -60, 1e-3, 1e4, 2.0 ** 40, 2.0 ** 41, -1.0, math.nan, math.inf, 1e-44, -0.0]
    b = Batch([2] * len(heat), 501, heat=heat, seed=4)
    accepted, following = b.check()
    assert following[6:10] == [-1] * 4 and accepted[6:10] == [1] * 4
    assert all(x >= 0 for x in following[:6] + following[10:])


def test_large_logits():
    """Differences past an exponential's range and past fp32's, and all logits of one size."""
    b = Batch([2] * 5, 600, heat=[1.0, 1.0, 0.5, 100.0, 1e-9], seed=5)
    b.z[0:2] *= 2e37
    b.z[2:4] += 1e6
    b.z[4:6] = -1e25 * (1.0 + b.z[4:6].abs())
    b.z[6:8] -= 3e4
    b.check()


def test_drafts_that_are_none():
    for probs in (False, True):
        b = Batch([3, 2, 2], 300, probs=probs, seed=6)
        b.tokens.copy_(_i32([0, -1, 4, 9, 300, 2 ** 31 - 1, -2 ** 31]))
        accepted, _ = b.check()
        assert accepted == [1, 1, 1]


def test_where_nothing_is_left_beside_the_draft():
    """p = q exactly, u at its largest: the draft stands or the draw is p's own."""
    for vocab in (64, 5000):
        b = Batch([2], vocab, probs=True, seed=7)
        b.z[0] = 0.0
        b.probs[0] = 1.5 / vocab  # (p - q < 0 everywhere)
        b.u[0] = 0.9
        b.tokens[1] = 3
        accepted, following, _ = b.call()
        assert accepted == [1] and following == [int(b.race[0].argmin())]
        b.probs = None  # a certain draft of a row that has no other
        b.z[0] = -math.inf
        b.z[0, 9] = 1.0
        b.tokens[1] = 9
        accepted, following, p = b.call()
        assert accepted == [2] and p[0] == 1.0


def test_refused_requests_and_rows_behind_the_last():
    b = Batch([4, 3, 2, 5], 333, seed=8)
    b.rows = paged.PageRows(_i32([0, 4, 7, 9, 30]), _i32([14, 0, 1, 40]))  # refused, shorter than its rows, past the arrays
    v = verify.DraftVerifier(40, 4)
    p = torch.full((14,), 7.0, device="cuda")
    a, x = v.verify(b.z, b.tokens, b.rows, uniforms=b.u, race=b.race, target_probs=p)
    m = next(b.models())
    assert m.allows(int(a[0]), int(x[0]))
    assert a.tolist()[1:] == [0, 0, 0] and x.tolist()[1:] == [-1] * 3
    assert p[4:].tolist() == [0.0] * 10
    b.rows = paged.PageRows(_i32([0, 4, 7, 9, 11]), _i32([14, 20, 20, 20]))  # three rows more than the requests have
    p.fill_(7.0)
    v.verify(b.z, b.tokens, b.rows, uniforms=b.u, race=b.race, target_probs=p)
    assert p[11:].tolist() == [7.0] * 3 and not bool((p[:11] == 7.0).any())
    empty = paged.PageRows(_i32([0, 0, 0]), _i32([0, 5]))
    a, x = v.verify(b.z[:0], b.tokens[:0], empty, uniforms=b.u[:0], race=b.race)
    assert a.tolist() == [0, 0] and x.tolist() == [-1, -1]


def test_lengths_that_are_no_lengths_stay_inside_the_arrays():
    b = Batch([4, 3, 2, 5], 333, seed=8)
    for start in ([0, -4, 7, 9, 14], [5, 4, 3, 2, 1], [-9, -7, -5, -3, -1], [2 ** 31 - 1] * 5, [0, 2 ** 31 - 1, 3, 9, 14]):
        b.rows = paged.PageRows(_i32(start), _i32([50] * 4))
        b.call()


@pytest.mark.parametrize("probs", [False, True])
def test_tokens_are_distributed_as_the_target_draws_them(probs):
    """4096 requests of the same row, drafts drawn from q (or the same one): the first token, be it the draft or its
    replacement, is distributed as p.  chi^2 of 7 degrees of freedom passes 45 once in 10^7 times."""
    vocab, n = 8, 4096
    g = torch.Generator(device="cuda").manual_seed(11)
    z = torch.randn(vocab, device="cuda", generator=g)
    q = torch.softmax(torch.randn(vocab, device="cuda", generator=g), -1)
    v = verify.DraftVerifier(2 * n, n)
    rows = paged.PageRows(_i32(list(range(0, 2 * n + 1, 2))), _i32([9] * n))
    draft = torch.multinomial(q.expand(n, vocab), 1, generator=g).flatten() if probs else torch.full((n,), 2, device="cuda")
    tokens = torch.stack([torch.zeros_like(draft), draft], 1).flatten().int()
    a, x = v.verify(z.repeat(2 * n, 1), tokens, rows, uniforms=torch.rand(2 * n, device="cuda", generator=g),
                    race=torch.empty(n, vocab, device="cuda").exponential_(generator=g),
                    draft_probs=q.repeat(2 * n, 1) if probs else None)
    p = torch.softmax(z.double(), -1)
    for first in (torch.where(a == 2, draft, x.long()), x.long()[a == 2]):  # the first token, and the one after drafts that stand
        count = torch.bincount(first, minlength=vocab).double()
        want = p * count.sum()
        assert float(((count - want).square() / want).sum()) < 45.0


def test_streams_graphs_and_two_verifiers():
    one, two = Batch([4, 1, 7], 5000, "bf16", True, [0.7, 1.0, 0.0], seed=12), Batch([2] * 30, 900, "f32", seed=13)
    v, w = verify.DraftVerifier(80, 40), verify.DraftVerifier(80, 40)
    want = [b.call(v)[:2] for b in (one, two)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):  # two calls at once, on two verifiers and streams
        a1 = v.verify(one.z, one.tokens, one.rows, one.u, one.race, one.heat, one.probs)
        a2 = w.verify(two.z, two.tokens, two.rows, two.u, two.race, stream=side)
    torch.cuda.synchronize()
    assert [t.tolist() for t in a1] == list(want[0]) and [t.tolist() for t in a2] == list(want[1])
    out = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2)]
    kw = dict(uniforms=one.u, race=one.race, temperature=one.heat, draft_probs=one.probs, accepted=out[0], next_tokens=out[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        v.verify(one.z, one.tokens, one.rows, **kw)
    for seed in (20, 21):
        other = Batch([1, 8, 3], 5000, "bf16", True, [0.0, 1.1, 0.6], seed=seed)
        for x in ("z", "tokens", "u", "race", "heat", "probs"):
            getattr(one, x).copy_(getattr(other, x))
        one.rows.row_start.copy_(other.rows.row_start)
        one.rows.seq_len.copy_(other.rows.seq_len)
        g.replay()
        assert [t.tolist() for t in out] == list(other.check())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_arguments_are_taken_alike_in_c_and_in_python(dtype, monkeypatch):
    b = Batch([4, 2], 300, dtype, True, [0.5, 1.0], seed=15, pad=3)
    want = [b.call(), b.call(draft_probs=None), b.call(temperature=None, uniforms=None, race=None, draft_probs=None)]
    for native in (True, False):
        v = verify.DraftVerifier(6, 2)
        if not native:
            monkeypatch.setattr(v, "_verify", None)
        got = [b.call(v), b.call(v, draft_probs=None), b.call(v, temperature=None, uniforms=None, race=None, draft_probs=None)]
        for x, y in zip(got, want):
            assert x[:2] == y[:2] and bool((x[2] == y[2]).all())
    v = verify.DraftVerifier(6, 2)
    v.close()
    with pytest.raises(cllm.CllmError):
        b.call(v)


@pytest.mark.parametrize("native", [True, False])
def test_refusals(native, monkeypatch):
    b = Batch([4, 2], 100, seed=14)
    v = verify.DraftVerifier(6, 2)
    if not native:
        monkeypatch.setattr(v, "_verify", None)
    ok = dict(logits=b.z, tokens=b.tokens, rows=b.rows, uniforms=b.u, race=b.race)
    out = torch.full((2,), 5, dtype=torch.int32, device="cuda")
    for bad in (dict(logits=b.z.double()), dict(logits=b.z[0]), dict(logits=b.z.cpu()), dict(logits=b.z.T), dict(tokens=b.tokens.long()),
                dict(tokens=b.tokens[:5]), dict(uniforms=b.u[:5]), dict(uniforms=b.u.double()), dict(race=b.race[:1]),
                dict(race=b.race[:, :99]), dict(race=b.race.half()), dict(temperature=torch.ones(1, device="cuda")),
                dict(temperature=torch.ones(2)), dict(draft_probs=b.race), dict(accepted=out[:1]), dict(next_tokens=out.long()),
                dict(target_probs=b.u[:5])):
        with pytest.raises(ValueError):
            v.verify(**{**ok, "accepted": out, **bad})
    big = Batch([5, 2], 100, seed=14)
    three = Batch([1, 1, 1], 100, seed=14)
    for bad in (dict(uniforms=None), dict(race=None), dict(uniforms=None, race=None, temperature=torch.ones(2, device="cuda")),
                dict(uniforms=None, race=None, draft_probs=b.z), dict(logits=big.z, tokens=big.tokens, rows=big.rows, uniforms=big.u),
                dict(logits=three.z, tokens=three.tokens, rows=three.rows, race=three.race, accepted=None),
                dict(logits=torch.zeros(1, 100, device="cuda").expand(6, 100))):
        with pytest.raises(cllm.CllmError) as e:
            v.verify(**{**ok, "accepted": out, **bad})
        assert e.value.status == -1
    assert out.tolist() == [5, 5]
    v.close()
    v.close()


def test_offsets_past_31_bits():
    """17000 rows of 131072 logits: the last request begins past 2^31 values."""
    vocab, n = 131072, [16990, 6, 4]
    g = torch.Generator(device="cuda").manual_seed(16)
    z = torch.zeros(sum(n), vocab, device="cuda", dtype=torch.bfloat16)
    first = [0, 16990, 16996]
    for r in [0, 1, *range(16990, 17000)]:
        z[r] = torch.randn(vocab, device="cuda", generator=g)
    tokens = torch.randint(0, vocab, (sum(n),), device="cuda", generator=g).int()
    for r in (16990, 16991, 16996):
        z[r, int(tokens[r + 1])] = 60.0
    u = torch.rand(sum(n), device="cuda", generator=g)
    race = torch.empty(3, vocab, device="cuda").exponential_(generator=g)
    rows = paged.PageRows(_i32([0, 16990, 16996, 17000]), _i32([20000] * 3))
    v = verify.DraftVerifier(17000, 3)
    for greedy in (False, True):
        p = torch.full((17000,), 7.0, device="cuda")
        a, x = v.verify(z, tokens, rows, target_probs=p, **({} if greedy else dict(uniforms=u, race=race)))
        for b, r in enumerate(first):
            m = Model(z[r:r + 6].double().cpu().numpy(), tokens[r:r + 6].tolist(), None if greedy else race[b].cpu().numpy(), u[r:r + 6].tolist())
            assert m.allows(int(a[b]), int(x[b]))
        assert a.tolist()[1:] == [3, 2] and not bool((p == 7.0).any())


def test_a_vocabulary_of_2_to_the_26():
    vocab = 2 ** 26 + 3
    g = torch.Generator(device="cuda").manual_seed(17)
    z = torch.randn(2, vocab, device="cuda", generator=g).half()
    z[0, vocab - 1] = 30.0
    race = torch.empty(1, vocab, device="cuda").exponential_(generator=g)
    rows, v, p = paged.PageRows(_i32([0, 2]), _i32([2])), verify.DraftVerifier(2, 1), torch.zeros(2, device="cuda")
    tokens = _i32([5, vocab - 1])
    a, x = v.verify(z, tokens, rows, uniforms=torch.tensor([0.5, 0.5], device="cuda"), race=race, target_probs=p)
    true = torch.softmax(z[0].double(), -1)[-1]
    assert abs(float(p[0]) - float(true)) <= 2 * TOL * float(true)
    ratio = z[1].double() - race[0].double().log()
    assert a.tolist() == [2] and float(ratio[x[0]]) >= float(ratio.max()) - 1e-5
    assert v.verify(z, tokens, rows)[0].tolist() == [2]
