"""A small server over the paged cache: requests come and go, prompts and Jacobi
blocks share each step's batch, and pages pass from one request to the next.

    python examples/paged_serving.py [--requests 12] [--slots 4] [--block 8] [--dtype f32]

Every step of the loop is ``paged.plan`` (pages, slots and positions of the step's
rows), then per layer ``PagedCache.append`` (rotary embedding, K and V into their pages)
and ``PagedCache.attention``; torch supplies the projections of the small decoder.
A request's first step is its prompt; after it every step verifies a block of n
tokens (Sec. 3.1: the longest prefix that reproduces itself is committed, the block
keeps the predictions that follow it and is filled with guesses).  The tokens are the
greedy ones, whatever the guesses and whoever shares the batch.
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import replace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2403_00835_gb300 import paged  # noqa: E402
from paper_2403_00835_gb300 import synthetic as syn  # noqa: E402


class PagedDecoder:
    """A LLaMA-style decoder over paged K and V, for batches of ragged rows."""

    def __init__(self, cfg, weights, n_pages, page_size, max_batch, max_rows, max_len):
        self.cfg, self.w = cfg, weights
        dt, dev = weights["tok_emb"].dtype, weights["tok_emb"].device
        pools = [torch.empty(cfg.n_layers, n_pages, cfg.n_kv_heads, page_size, cfg.head_dim, dtype=dt, device=dev) for _ in range(2)]
        self.cache = paged.PagedCache(*pools, cfg.n_heads)
        self.tables = paged.PageTables.empty(n_pages, page_size, max_batch, -(-max_len // page_size), dev)
        self.rows = paged.PageRows.empty(max_batch, max_rows, dev)
        i = torch.arange(cfg.head_dim // 2, dtype=torch.float64, device=dev)
        ang = torch.arange(max_len, dtype=torch.float64, device=dev)[:, None] * float(cfg.rope_theta) ** (-2.0 * i / cfg.head_dim)
        self.rope = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()
        # one product gives q, k and v of a row side by side
        self.wqkv = [torch.cat([weights[k][layer] for k in ("wq", "wk", "wv")]) for layer in range(cfg.n_layers)]

    def _norm(self, x, gain):
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.cfg.rms_eps)).to(gain.dtype) * gain

    def plan(self, ctx, new):
        paged.plan(self.tables, self.rows, ctx, new)

    def forward(self, tokens):
        """Predictions after every row of the planned step."""
        c, w = self.cfg, self.w
        t, dq, dkv = tokens.numel(), c.n_heads * c.head_dim, c.n_kv_heads * c.head_dim
        x = w["tok_emb"][tokens].float()
        for layer in range(c.n_layers):
            qkv = self._norm(x, w["attn_norm"][layer]) @ self.wqkv[layer].T
            q, k, v = (s.unflatten(1, (-1, c.head_dim)) for s in qkv.split([dq, dkv, dkv], 1))
            self.cache.append(layer, k, v, self.rows.slots, q=q, rope=self.rope, positions=self.rows.positions)
            o = self.cache.attention(layer, q, self.rows, self.tables, out=torch.empty(t, c.n_heads, c.head_dim, dtype=q.dtype, device=q.device))
            x = x + (o.view(t, dq) @ w["wo"][layer].T).float()
            h = self._norm(x, w["mlp_norm"][layer])
            x = x + ((torch.nn.functional.silu(h @ w["w_gate"][layer].T) * (h @ w["w_up"][layer].T)) @ w["w_down"][layer].T).float()
        return (self._norm(x, w["final_norm"]) @ w["lm_head"].T).argmax(-1)


class Request:
    def __init__(self, prompt, max_new, n, rng, vocab):
        self.prompt, self.max_new, self.n, self.rng, self.vocab = prompt, max_new, n, rng, vocab
        self.cached, self.out, self.block, self.steps = 0, [], None, 0

    def rows(self):
        return self.prompt if self.block is None else self.block

    def take(self, predictions):
        """The predictions after this step's rows; True when the request has ended."""
        if self.block is None:
            a, head = len(self.prompt), predictions[-1]
            kept = []
        else:
            a = 1
            while a < self.n and self.block[a] == predictions[a - 1]:
                a += 1
            self.out += self.block[:a]
            head, kept = predictions[a - 1], predictions[a:]
            self.steps += 1
        self.cached += a
        self.block = [head] + kept + self.rng.integers(0, self.vocab, self.n - 1 - len(kept)).tolist()
        return len(self.out) >= self.max_new


def serve(cfg, weights, prompts, max_new, n=8, slots=4, page_size=16, n_pages=None, seed=0):
    """Tokens of every prompt ([max_new] each), and the steps run.  Prompts wait for a
    free slot, and for pages when the pool is small."""
    dev = weights["tok_emb"].device
    longest = max(len(p) for p in prompts) + max_new + 2 * n
    need = -(-longest // page_size)
    n_pages = n_pages or need * slots
    max_rows = slots * max(n, max(len(p) for p in prompts))
    dec = PagedDecoder(cfg, weights, n_pages, page_size, slots, max_rows, need * page_size)
    rng = np.random.default_rng(seed)
    waiting = [Request(p, max_new, n, rng, cfg.vocab) for p in prompts]
    everyone, running, steps, stalled = list(waiting), [None] * slots, 0, 0
    while waiting or any(running):
        for i in range(slots):
            if running[i] is None and waiting:
                running[i] = waiting.pop(0)
        ctx = [r.cached if r else 0 for r in running]  # an ended request (0, 0) gives its pages back
        new = [len(r.rows()) if r else 0 for r in running]
        dec.plan(torch.tensor(ctx, dtype=torch.int32, device=dev), torch.tensor(new, dtype=torch.int32, device=dev))
        tokens = torch.tensor(sum((r.rows() for r in running if r), []), device=dev)
        predictions = dec.forward(tokens).tolist()
        granted = dec.rows.granted.tolist()
        at = 0
        for i, r in enumerate(running):
            if r is None:
                continue
            mine = predictions[at:at + new[i]]
            at += new[i]
            if granted[i] and r.take(mine):  # (refused: the same rows again, when pages have come back)
                running[i] = None
        # (pages that a step gave back can be handed out in the next)
        stalled = 0 if any(g for g, m in zip(granted, new) if m) else stalled + 1
        if stalled > 1:
            raise RuntimeError("the pool is too small for the running requests")
        steps += 1
    dec.cache.check()
    return [r.out[:max_new] for r in everyone], steps


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--slots", type=int, default=4)
    ap.add_argument("--block", type=int, default=8)
    ap.add_argument("--max-new", type=int, default=32)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    torch.backends.cuda.matmul.allow_tf32 = False
    cfg = replace(syn.TINY, dtype=a.dtype)
    w = syn.make_weights(cfg, seed=0, device="cuda")
    prompts = syn.make_prompts(cfg.vocab, syn.ragged_lens(a.requests, 5, 90, seed=3), seed=1)
    out, steps = serve(cfg, w, prompts, a.max_new, n=a.block, slots=a.slots)
    for p, o in zip(prompts, out):
        print(f"prompt of {len(p):3d}: {o[:12]} ...")
    print(f"{sum(map(len, out))} tokens in {steps} steps of up to {a.slots} requests")


if __name__ == "__main__":
    main()
