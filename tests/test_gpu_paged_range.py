"""fp16 probabilities far below a row's largest: a context of equally small ones under one
high score (a long context with a sink token) keeps its weight."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged
from tests.paged_util import ROUND, Step

pytestmark = pytest.mark.gpu


# every 16-bit kernel: few rows, 4 bands, 2 bands, one slot's rows, both slots'
@pytest.mark.parametrize("heads,kv,new", [(8, 2, 3), (24, 1, 1), (40, 1, 1), (4, 1, 25), (40, 40, 130)])
@pytest.mark.parametrize("high", [16.5, 17.75, 20.0])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_small_probabilities_under_one_high_score(dtype, heads, kv, new, high):
    batch = 4 if new > 100 else 1
    step = Step([700] * batch, [new] * batch, heads, kv, 64, 16, dtype, seed=new)
    step.q.zero_()
    step.q[:, :, 0] = 1.0
    for b in range(batch):
        pages = step.table[b].long()
        step.k[0, pages] = 0.0       # (what lies past the request is not seen)
        step.v[0, pages] = 1.0
        step.token(step.k, b, 0)[:, 0] = high
        step.token(step.v, b, 0)[...] = 0.0
    cache = paged.PagedCache(step.k, step.v, heads)
    got = cache.attention(0, step.q, paged.PageRows(step.row_start, step.seq_len), paged.PageTables(step.table, page_size=16),
                          scale=1.0)
    cache.check()
    o, _, ab, delta = step.attention(scale=1.0)
    u32, u, n = ROUND["f32"], ROUND[dtype], 700 + new
    # a score's 68 terms (change of base among them), the exponential, sums of n terms, the
    # rounding of a probability: relative.  fp16 below its normal range rounds to a multiple of
    # 2^-24: half of that, of a largest probability of 2^7 or more; and in the result itself.
    rel = 2 * 68 * u32 * delta + 2.0 ** -21 + 2 * (n + 8) * u32 + u
    tol = rel[..., None] * ab + u * o.abs()
    if dtype == "f16":
        tol = tol + 2.0 ** -32 * n + 2.0 ** -25
    assert float(o.max()) > 20 * 2.0 ** -25  # (the result is not lost in its own rounding)
    assert bool(((got.double() - o).abs() <= tol).all()), float(((got.double() - o).abs() / tol).max())
