"""Shared helpers of the paged-cache tests: random steps, and the operators'
definitions in fp64 (numpy-free torch on the CPU or GPU, one row at a time)."""
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {n: torch.finfo(t).eps / 2 for n, t in DTYPES.items()}  # unit roundoff


class Step:
    """One step of a batch on random pages.  Everything in the pools that is not
    a token of a request is NaN, and table entries past a request's pages are -1."""

    def __init__(self, ctx, new, heads, kv_heads, hd, page, dtype, order="page", seed=0, layers=1, spare=3, width=None,
                 n_pages=None, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.ctx, self.new, self.heads, self.kv_heads, self.hd, self.page, self.dtype = ctx, new, heads, kv_heads, hd, page, dtype
        dt = DTYPES[dtype]
        total = [c + n for c, n in zip(ctx, new)]
        used = [-(-t // page) for t in total]
        self.n_pages = n_pages or sum(used) + spare
        self.width = width or max(1, max(used))
        pages = rng.permutation(self.n_pages)
        shape = (layers, self.n_pages, kv_heads, page, hd) if order == "page" else (layers, self.n_pages, page, kv_heads, hd)
        self.k, self.v = (torch.empty(shape, dtype=dt, device=device) for _ in range(2))
        if n_pages is None:
            self.k.fill_(float("nan"))
            self.v.fill_(float("nan"))
        if order == "token":
            self.k, self.v = self.k.transpose(2, 3), self.v.transpose(2, 3)
        self.layer = layers - 1
        table = np.full((len(ctx), self.width), -1, np.int32)
        at = 0
        for b, (t, u) in enumerate(zip(total, used)):
            mine = pages[at:at + u] if n_pages is None else np.arange(self.n_pages - at - u, self.n_pages - at)
            at += u
            table[b, :u] = mine
            for i, p in enumerate(mine.tolist()):
                m = min(page, t - i * page)
                for pool in (self.k, self.v):
                    if n_pages is not None:
                        pool[self.layer, p] = float("nan")
                    pool[self.layer, p, :, :m] = torch.randn(kv_heads, m, hd, generator=gen, device=device).to(dt)
        self.table = torch.from_numpy(table).to(device)
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.row_start = torch.from_numpy(start).to(device)
        self.seq_len = torch.tensor(total, dtype=torch.int32, device=device)
        self.rows = int(start[-1])
        self.q = (1.5 * torch.randn(self.rows, heads, hd, generator=gen, device=device)).to(dt)

    def token(self, pool, b, pos):
        """A view of one token's heads in a pool."""
        p = int(self.table[b, pos // self.page])
        return pool[self.layer, p, :, pos % self.page]

    def gathered(self, pool, b, length):
        pages = self.table[b, :-(-length // self.page)].long()
        return pool[self.layer][pages].transpose(1, 2).reshape(-1, self.kv_heads, self.hd)[:length].double()

    def attention(self, scale=None, window=0, mask=None, seq_len=None):
        """(out, lse, sum p |v|, largest score error's scale) in fp64.  mask: bool
        [rows][new tokens of the longest request] or None."""
        scale = self.hd ** -0.5 if scale is None else scale
        dev = self.q.device
        o = torch.zeros(self.rows, self.heads, self.hd, dtype=torch.float64, device=dev)
        ab = torch.zeros_like(o)
        lse = torch.full((self.rows, self.heads), -math.inf, dtype=torch.float64, device=dev)
        delta = torch.zeros_like(lse)
        g = self.heads // self.kv_heads
        lens = self.seq_len.tolist() if seq_len is None else seq_len
        starts = self.row_start.tolist()
        for b, n in enumerate(self.new):
            ctx = lens[b] - n
            if n == 0 or ctx < 0:
                continue
            k, v = self.gathered(self.k, b, lens[b]), self.gathered(self.v, b, lens[b])
            pos = torch.arange(lens[b], device=dev)
            for i in range(n):
                r = starts[b] + i
                if mask is None:
                    see = pos <= ctx + i
                else:
                    see = torch.cat([torch.ones(ctx, dtype=torch.bool, device=dev), mask[r, :n].to(dev)])
                if window:
                    see = see & (ctx + i - pos < window)
                if not bool(see.any()):
                    continue
                kk, vv = k[see].repeat_interleave(g, 1), v[see].repeat_interleave(g, 1)  # [keys][H][hd]
                qr = self.q[r].double()
                s = torch.einsum("hd,khd->hk", qr, kk) * scale
                lse[r] = torch.logsumexp(s, -1)
                p = (s - lse[r][:, None]).exp()
                o[r] = torch.einsum("hk,khd->hd", p, vv)
                ab[r] = torch.einsum("hk,khd->hd", p, vv.abs())
                delta[r] = (torch.einsum("hd,khd->hk", qr.abs(), kk.abs()) * scale).amax(-1)
        return o, lse, ab, delta

    def bound(self, ab, delta, o):
        """How far a kernel may be from fp64 (per element of out, and of lse).

        A score is a sum of hd products: off by at most hd u32 sum |q k| scale, and
        by 4 u32 of itself for the change of base; a probability by that, the
        exponential's 2^-21, and its rounding to the pools' type (16-bit pools; in
        fp16 also 2^-25 of the row's largest, for those below its normal range);
        sums of n terms in fp32 by n u32 of their terms' size; the result by its rounding."""
        u32, u = ROUND["f32"], ROUND[self.dtype]
        n = max(c + m for c, m in zip(self.ctx, self.new))
        ds = (self.hd + 4) * u32 * delta
        rel = 2 * ds + 2.0 ** -21 + 2 * (n + 8) * u32 + (u if self.dtype != "f32" else 0.0)
        tol = rel[..., None] * ab + u * o.abs()
        if self.dtype == "f16":
            big = torch.nan_to_num(self.v.abs(), nan=0.0, posinf=0.0).max().double()
            tol = tol + 2.0 ** -25 * n * big
        return tol + 1e-30, ds + 2.0 ** -21 + (n + 8) * u32 + 2.0 ** -22 * delta


def pack_mask(see):
    """bool [rows][n] -> int32 words [rows][ceil(n / 32)]."""
    rows, n = see.shape
    words = -(-max(n, 1) // 32)
    out = np.zeros((rows, words), np.uint32)
    s = see.cpu().numpy()
    for j in range(n):
        out[:, j // 32] |= s[:, j].astype(np.uint32) << np.uint32(j % 32)
    return torch.from_numpy(out.view(np.int32)).to("cuda" if torch.cuda.is_available() else "cpu")


class TablesModel:
    """Page plan, one request after the other on Python lists."""

    def __init__(self, n_pages, page, max_batch, width):
        self.n_pages, self.page, self.width = n_pages, page, width
        self.tables = [[] for _ in range(max_batch)]
        self.ring, self.head, self.count = list(range(n_pages)), 0, n_pages

    def plan(self, ctx, new, max_rows):
        row_start, granted, back, taken = [0], [], [], 0
        slots, positions = [-1] * max_rows, [0] * max_rows
        wanted = 0
        for b, (c, n) in enumerate(zip(ctx, new)):
            t0 = row_start[-1]
            row_start.append(min(t0 + max(n, 0), 2 ** 31 - 1))
            t = self.tables[b]
            ok = c >= 0 and n >= 0 and c + n <= self.width * self.page and row_start[-1] <= max_rows
            need = -(-(c + n) // self.page) if ok else len(t)
            grow = max(need - len(t), 0)
            wanted += grow
            if grow and wanted > self.count:
                ok = False
            granted.append(int(ok))
            if not ok:
                continue
            for _ in range(grow):
                t.append(self.ring[(self.head + taken) % self.n_pages])
                taken += 1
            back += t[need:]
            del t[need:]
            for i in range(n):
                p = c + i
                slots[t0 + i], positions[t0 + i] = t[p // self.page] * self.page + p % self.page, p
        for r, p in enumerate(back):
            self.ring[(self.head + self.count + r) % self.n_pages] = p
        self.head, self.count = (self.head + taken) % self.n_pages, self.count - taken + len(back)
        seq = [c + n if g else 0 for c, n, g in zip(ctx, new, granted)]
        return dict(row_start=row_start, granted=granted, seq_len=seq, slots=slots, positions=positions)
