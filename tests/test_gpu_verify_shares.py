"""Draft verification where a row's or a race's vocabulary is cut differently: warps of one small CTA (4099), of one large
one (20011), warps all over the GPU whose shares meet in memory (50021; 4099 with many rows).  Ties, values
that are no numbers, masked stretches and races without weights, each within one share or across several;
calls one after another on one verifier, whose counters the last of a row's or a race's warps has to leave at zero."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged, verify
from tests.test_gpu_verify import Batch, _i32

pytestmark = pytest.mark.gpu

VOCABS = [4099, 20011, 50021]
DTYPES = ["f32", "bf16", "f16"]


def _again(b, v, want, times=3, **kw):
    """The same answers in later calls on the verifier."""
    for _ in range(times):
        assert b.call(v, **kw)[:2] == tuple(want)


GREEDY = dict(uniforms=None, race=None, temperature=None, draft_probs=None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_ties_in_different_shares(dtype, vocab):
    """Equal logits (greedy) and equal ratios (a race of ones) at both ends, in the middle, and next to one another."""
    places = [[0, vocab - 1], [vocab - 2, vocab - 1], [vocab // 2, vocab // 2 + 1], [1023, 1024], [vocab // 3, 2 * vocab // 3],
              list(range(7, vocab, 1000))]
    b = Batch([2] * len(places), vocab, dtype, seed=1)
    b.z.zero_()
    for i, at in enumerate(places):
        b.z[2 * i, at] = 3.0
        b.tokens[2 * i + 1] = at[-1] if i % 2 else at[0]
    b.z[1::2] = -2.0
    first = [1 if i % 2 else 2 for i in range(len(places))]
    want = (first, [at[0] if i % 2 else 0 for i, at in enumerate(places)])
    v = verify.DraftVerifier(b.t, len(places))
    assert b.check(greedy=True, verifier=v) == want
    _again(b, v, want, **GREEDY)
    b.race.fill_(1.0)
    b.u.fill_(0.999)
    want = ([1] * len(places), [at[0] if i % 2 else at[1] for i, at in enumerate(places)])
    assert b.check(verifier=v) == want
    _again(b, v, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_one_bad_logit_in_any_share(dtype, vocab, bad):
    """The fourth row of each request has it, in another place; its drafts stand up to there."""
    places = [0, 1, 8, 1000, 1023, 1024, vocab // 2, vocab - 1030, vocab - 9, vocab - 2, vocab - 1]
    b = Batch([6] * len(places), vocab, dtype, seed=2, peak=60.0 if dtype != "f16" else 30.0)
    b.tokens[1:] = b.z.argmax(-1)[:-1].int()
    for i, at in enumerate(places):
        b.z[6 * i + 3, at] = bad
    v = verify.DraftVerifier(b.t, len(places))
    want = [4] * len(places), [-1] * len(places)
    assert b.check(verifier=v) == want
    _again(b, v, want)
    greedy = b.check(greedy=True, verifier=v)
    if math.isnan(bad):
        assert greedy == want
    else:
        assert greedy == (want[0], places)
    _again(b, v, greedy, **GREEDY)
    b.heat = torch.tensor([0.0, 1.0] * 6, device="cuda")[:len(places)].contiguous()
    b.check(verifier=v)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("probs", [False, True])
def test_stretches_of_masked_logits(dtype, vocab, probs):
    """Rows of which only a stretch, or one value, is above -inf; none at all ends a request."""
    keep = [(0, vocab), (0, 5), (vocab - 3, vocab), (vocab // 2, vocab // 2 + 1), (1000, 3000), (vocab - 2000, vocab - 40), (0, 0), (0, 1)]
    b = Batch([3] * len(keep), vocab, dtype, probs, seed=3)
    at = torch.arange(vocab, device="cuda")
    for i, (lo, hi) in enumerate(keep):
        b.z[3 * i:3 * i + 3, (at < lo) | (at >= hi)] = -math.inf
    v = verify.DraftVerifier(b.t, len(keep))
    accepted, following = b.check(verifier=v)
    for (lo, hi), x in zip(keep, following):
        assert lo <= x < hi or (hi == 0 and x == -1)
    _again(b, v, (accepted, following))
    accepted, following = b.check(greedy=True, verifier=v)
    for (lo, hi), x in zip(keep, following):
        assert lo <= x < hi or (hi == 0 and x == -1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("probs", [False, True])
def test_greedy_and_sampled_requests_in_one_call(dtype, vocab, probs):
    n = [1, 5, 0, 8, 2, 0, 9, 3]
    b = Batch(n, vocab, dtype, probs, [0.0, 1.0, 0.7, 0.0, 1.3, 0.0, 0.5, 0.0], seed=4, pad=3)
    v = verify.DraftVerifier(b.t, len(n))
    want = b.check(verifier=v)
    _again(b, v, want)


@pytest.mark.parametrize("vocab", VOCABS)
def test_races_without_weights(vocab):
    """p - q < 0 everywhere: the draw is p's own, by one warp over the whole vocabulary, after parts that found nothing."""
    b = Batch([2] * 6, vocab, probs=True, seed=5)
    b.z[0::2] = 0.0
    b.probs[0::2] = 1.5 / vocab
    b.u[0::2] = 0.9
    b.tokens[1::2] = 3
    v = verify.DraftVerifier(b.t, 6)
    want = [1] * 6, b.race.argmin(-1).tolist()
    assert b.call(v)[:2] == want
    _again(b, v, want)
    for x in b.z[0::2]:
        x.fill_(-math.inf)
        x[vocab - 7] = 1.0
    b.probs = None
    b.tokens[1::2] = vocab - 7
    accepted, following, p = b.call(v)
    assert accepted == [2] * 6 and (p[0::2] == 1.0).all()
    b.check(verifier=v)


@pytest.mark.parametrize("vocab", VOCABS)
def test_drafts_that_are_none(vocab):
    b = Batch([3, 2, 2, 2], vocab, probs=True, seed=6)
    b.tokens.copy_(_i32([0, -1, 4, 9, vocab, 0, 2 ** 31 - 1, 1, -2 ** 31]))
    v = verify.DraftVerifier(b.t, 4)
    want = b.check(verifier=v)
    assert want[0] == [1] * 4
    b.probs = None
    assert b.check(verifier=v) == want  # (drawn from p itself either way)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows_of_a_short_vocabulary(dtype):
    """More rows than the GPU holds small CTAs for: their shares meet in memory as well."""
    b = Batch([2] * 700, 4099, dtype, heat=[0.0, 1.0, 0.8, 1.2] * 175, seed=7)
    v = verify.DraftVerifier(b.t, 700)
    want = b.check(verifier=v)
    _again(b, v, want, times=2)


def test_calls_of_all_kinds_on_one_verifier():
    """Shapes that cut rows and races differently, refused and empty requests between: every call answers as on a new verifier."""
    kinds = [Batch([3, 4], 50021, "f32", True, seed=8), Batch([2] * 700, 4099, "f16", seed=9), Batch([5] * 12, 20011, "bf16", True, seed=10),
             Batch([1], 131071, "bf16", seed=11), Batch([4, 0, 9], 50021, "f16", heat=[0.0, 1.0, 1.0], seed=12), Batch([7] * 40, 4099, "f32", seed=13)]
    refused = Batch([4, 3, 2, 5], 50021, seed=14)
    refused.rows = paged.PageRows(_i32([0, 4, 7, 9, 30]), _i32([14, 0, 1, 40]))
    kinds.append(refused)
    want = [b.call() for b in kinds]
    v = verify.DraftVerifier(1400, 700)
    for order in (range(len(kinds)), range(len(kinds) - 1, -1, -1)):
        for i in order:
            got = kinds[i].call(v)
            assert got[:2] == want[i][:2] and (got[2] == want[i][2]).all()
            got = kinds[i].call(v, **GREEDY)
            assert got[:2] == kinds[i].call(**GREEDY)[:2]
