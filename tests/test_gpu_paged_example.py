"""The serving example over the paged cache: its tokens are the greedy ones of the
engine, however requests share steps and pages, and whatever the pool's size."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import synthetic as syn
from tests.parity_util import engine_for

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("slots,block,page,n_pages", [(1, 4, 16, None), (4, 8, 8, None), (3, 1, 32, None), (4, 8, 16, 13)])
def test_serving_gives_the_engines_greedy_tokens(slots, block, page, n_pages):
    import paged_serving
    cfg = syn.TINY
    w = syn.make_weights(cfg, seed=0, device="cuda")
    prompts = syn.make_prompts(cfg.vocab, [5, 40, 17, 1, 63, 33, 9], seed=1)
    eng = engine_for(cfg, w, 1, 160, 1)
    want = [eng.ar_decode([p], 20)[0].tolist() for p in prompts]
    eng.close()
    got, steps = paged_serving.serve(cfg, w, prompts, 20, n=block, slots=slots, page_size=page, n_pages=n_pages)
    assert got == want
    assert steps >= 20 * len(prompts) / slots / block
