"""A sampled decode over the paged cache with everything that a step has: plan, keys and queries
normalised and rotated by a scaled table, attention with a window and first tokens, verification of
drafts with a temperature.  Logits against a forward pass over all tokens from the definitions in fp64,
verdicts against the model; requests of several lengths that begin and end."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged, verify
from tests.verify_util import Model

pytestmark = pytest.mark.gpu

D, HEADS, KV, HD, LAYERS, VOCAB, PAGE, WINDOW, SINKS = 96, 4, 2, 64, 2, 211, 8, 13, 3
DIMS, FREQ, AMP = 32, paged.rope_frequencies(32, 1e4, "ramp", 4.0, trained=64), 0.1 * math.log(4.0) + 1.0


class Decoder:
    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return torch.randn(*shape, device="cuda", generator=g) / math.sqrt(shape[-1])

        self.emb = torch.randn(VOCAB, D, device="cuda", generator=g)
        self.qkv = [w((HEADS + 2 * KV) * HD, D) for _ in range(LAYERS)]
        self.out = [w(D, HEADS * HD) for _ in range(LAYERS)]
        self.head = 2.0 * w(VOCAB, D)
        self.gains = [[1.0 + 0.3 * torch.randn(HD, device="cuda", generator=g) for _ in "qk"] for _ in range(LAYERS)]

    def step(self, s, tokens):
        """Logits after every row of the planned step."""
        x = self.emb[tokens]
        for i in range(LAYERS):
            q, k, v = (t.unflatten(1, (-1, HD)) for t in (x @ self.qkv[i].T).split([HEADS * HD, KV * HD, KV * HD], 1))
            s.cache.append(i, k, v, s.rows.slots, q=q, rope=s.rope, positions=s.rows.positions, q_norm=self.gains[i][0],
                           k_norm=self.gains[i][1], eps=1e-5, interleaved=True)
            o = s.cache.attention(i, q, s.rows, s.tables, window=WINDOW, sinks=SINKS)
            x = x + o.flatten(1) @ self.out[i].T
        return x @ self.head.T

    def definition(self, tokens):
        """Logits after every token, in fp64, without a cache."""
        n = len(tokens)
        x = self.emb.double()[tokens]
        ang = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * torch.tensor(list(FREQ), dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.full_like(ang, AMP), ang)[:, None]
        at = torch.arange(n, device="cuda")
        gap = at[:, None] - at[None, :]
        see = (gap >= 0) & ((gap < WINDOW) | (at < SINKS)[None, :])

        def head(y, gain):
            y = y / (y.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gain.double()
            z = torch.view_as_complex(y[..., :DIMS].unflatten(-1, (-1, 2)).contiguous()) * turn
            return torch.cat([torch.view_as_real(z).flatten(-2), y[..., DIMS:]], -1)

        for i in range(LAYERS):
            q, k, v = (t.unflatten(1, (-1, HD)) for t in (x @ self.qkv[i].double().T).split([HEADS * HD, KV * HD, KV * HD], 1))
            q, k = head(q, self.gains[i][0]), head(k, self.gains[i][1]).repeat_interleave(HEADS // KV, 1)
            sc = torch.einsum("ihd,jhd->hij", q, k) * HD ** -0.5
            p = torch.softmax(sc.masked_fill(~see, -math.inf), -1)
            x = x + torch.einsum("hij,jhd->ihd", p, v.repeat_interleave(HEADS // KV, 1)).flatten(1) @ self.out[i].double().T
        return x @ self.head.double().T


class Server:
    def __init__(self, slots, pages, max_rows, longest):
        pools = [torch.full((LAYERS, pages, KV, PAGE, HD), float("nan"), device="cuda") for _ in range(2)]
        self.cache = paged.PagedCache(*pools, HEADS)
        self.tables = paged.PageTables.empty(pages, PAGE, slots, -(-longest // PAGE))
        self.rows = paged.PageRows.empty(slots, max_rows)
        self.verifier = verify.DraftVerifier(max_rows, slots)
        self.rope = paged.rope_table(longest, FREQ, AMP)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("seed,heat", [(0, [0.0, 0.7, 1.0]), (1, [1.3, 0.0, 0.5])])
def test_steps_of_a_sampled_decode(seed, heat):
    allow = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        _run(seed, heat)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = allow


def _run(seed, heat):
    rng = np.random.default_rng(seed)
    slots, block = 3, 5
    dec, s = Decoder(seed), Server(slots, pages=24, max_rows=80, longest=96)
    waiting = [rng.integers(0, VOCAB, n).tolist() for n in (1, 17, 30, 6, 2)]
    text = [None] * slots  # committed tokens, the head of the next block last
    drafts, cached = [[]] * slots, [0] * slots
    stood = finished = 0
    for step in range(80):
        for i in range(slots):
            if text[i] is None and waiting:
                text[i], drafts[i], cached[i] = list(waiting.pop()), [], 0
        if not any(text):
            break
        blocks = [[] if t is None else t[c:] + d for t, c, d in zip(text, cached, drafts)]
        paged.plan(s.tables, s.rows, _i32([c if t else 0 for t, c in zip(text, cached)]), _i32([len(b) for b in blocks]))
        tokens = torch.tensor(sum(blocks, []), device="cuda")
        t = len(tokens)
        logits = dec.step(s, tokens)
        u = torch.from_numpy(rng.random(t).astype(np.float32)).to("cuda")
        race = torch.from_numpy(rng.exponential(size=(slots, VOCAB)).astype(np.float32)).to("cuda")
        # (a prompt's tokens stand by themselves: its last row judges, and rows before do not)
        known = _i32([0 if x is None else len(x) - c - 1 for x, c in zip(text, cached)])
        start = s.rows.row_start
        # each request's rows from its head on: gathered, as a server with prompts in the batch would
        keep = torch.cat([torch.arange(int(start[i]) + int(known[i]), int(start[i + 1]), device="cuda") for i in range(slots)])
        n = [len(b) - int(k) for b, k in zip(blocks, known)]
        heads = paged.PageRows(_i32(np.concatenate([[0], np.cumsum(n)]).tolist()), s.rows.seq_len)
        accepted, following = s.verifier.verify(logits[keep], tokens[keep].int(), heads, uniforms=u[:len(keep)], race=race,
                                                temperature=torch.tensor(heat, device="cuda"))
        s.cache.check()
        accepted, following = accepted.tolist(), following.tolist()
        z, at, r0 = logits.double(), 0, 0
        for i in range(slots):
            if text[i] is None:
                assert (accepted[i], following[i]) == (0, -1)
                continue
            want = dec.definition(text[i] + drafts[i])[cached[i]:]
            mine = z[r0:r0 + len(blocks[i])]
            r0 += len(blocks[i])
            # some 300 fp32 sums of 64 to 256 terms a logit of size 5: 2^-24 * 256 * 5 * 4 at the worst
            assert float((mine - want).abs().max()) <= 3e-4
            m = Model(mine[-n[i]:].cpu().numpy(), tokens[keep][at:at + n[i]].tolist(), race[i].cpu().numpy(), u[at:at + n[i]].cpu().numpy(), heat[i])
            at += n[i]
            assert m.allows(accepted[i], following[i])
            stood += accepted[i] - 1
            text[i] += drafts[i][:accepted[i] - 1] + [following[i]]
            cached[i] = len(text[i]) - 1
            # the next drafts: what the target thinks likely after these rows, and guesses
            likely = mine.argmax(-1).tolist()
            drafts[i] = (likely[-n[i]:][accepted[i]:] + rng.integers(0, VOCAB, block).tolist())[:block - 1]
            if step % 3 == 0:  # now and then the right ones, so that some stand
                more = list(text[i])
                for _ in range(2):
                    more.append(int(dec.definition(more)[-1].argmax()))
                drafts[i][:2] = more[len(text[i]):]
            if len(text[i]) > 36:
                text[i], drafts[i], finished = None, [], finished + 1
    assert finished == 5 and stood > 5
