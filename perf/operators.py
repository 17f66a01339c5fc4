"""Performance cases of the paged key/value cache: the block tables and slot maps
of a step (``paged.plan``), the write of its keys and values with the rotary
embedding (``PagedCache.append``), and the attention of its new tokens over the
pages (``PagedCache.attention``).

``own`` false computes the same with elementary torch operations in fp32.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _plan(batch, page, lo, hi, new_lo, new_hi, done=0.0, short=0.0, name=None):
    """Requests with lo..hi cached tokens that get new_lo..new_hi more; a share
    `done` of them has ended and gives its pages back; `short`: the share of the
    pages wanted that the pool lacks."""
    c = dict(op="plan", batch=batch, page=page, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, done=done, short=short)
    return dict(c, name=name) if name else c


def _append(rows, heads, kv_heads, hd, page, dtype, order, rope=True, name=None):
    """order: "page" has a page's tokens of one head together, "token" one token's heads."""
    c = dict(op="append", rows=rows, heads=heads, kv_heads=kv_heads, hd=hd, page=page, dtype=dtype, order=order,
             rope=rope)
    return dict(c, name=name) if name else c


def _attn(batch, new, lo, hi, heads, kv_heads, hd, page, dtype, order="page", window=0, mask=False, name=None):
    """`new` tokens for each request after lo..hi cached ones."""
    c = dict(op="attention", batch=batch, new=new, lo=lo, hi=hi, heads=heads, kv_heads=kv_heads, hd=hd, page=page,
             dtype=dtype, order=order, window=window, mask=mask)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's request, the usual block of 16: launch latency
        _plan(1, 16, 128, 128, 16, 16, name="plan_one_block"),
        # a full server between two steps: ragged contexts, a tenth of the requests ended, prompts among the blocks
        _plan(512, 16, 0, 4096, 1, 128, done=0.1, name="plan_server_512"),
        # the keys and values of one block of 16
        _append(16, 32, 32, 128, 16, "f16", "page", name="append_block16"),
        # a batch of blocks, grouped heads, token-major pages
        _append(256, 32, 8, 128, 64, "bf16", "token", name="append_batch256"),
        # a chunk of prompts
        _append(8192, 32, 32, 128, 64, "f16", "page", name="append_prefill8192"),
        # the small fp32 decoder's block of 8
        _attn(1, 8, 32, 96, 4, 4, 64, 16, "f32", name="attn_tiny_f32_n8"),
        # one request of the 7B shape, the usual block of 16 after a prompt of 128
        _attn(1, 16, 128, 128, 32, 32, 128, 16, "f16", name="attn_7b_n16"),
        # the coder-style batch: ragged prompts, 256 rows
        _attn(8, 32, 256, 1024, 32, 32, 128, 32, "bf16", "token", name="attn_coder_batch8_n32"),
        # verification of several candidate n-grams at once: a mask among 61 new tokens, grouped heads
        _attn(4, 61, 700, 1100, 32, 8, 128, 64, "f16", mask=True, name="attn_verify_n61"),
        # greedy decoding of a full batch: one token a request
        _attn(16, 1, 4096, 4096, 32, 8, 128, 64, "bf16", name="attn_ar_batch16"),
        # a block of 16 far into a very long context
        _attn(1, 16, 131072, 131072, 32, 8, 128, 128, "f16", name="attn_long_131072"),
        # a chunk of a long prompt
        _attn(1, 2048, 4096, 4096, 32, 32, 128, 64, "bf16", name="attn_chunk2048"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    u = rng.random()
    if u < 0.2:
        lo = rng.choice((0, 1, _log_int(rng, 1, 2000)))
        new_lo = rng.choice((0, 1, _log_int(rng, 1, 32)))
        return _plan(_log_int(rng, 1, 512), 1 << rng.randint(3, 8), lo, max(lo, _log_int(rng, 1, 4000)), new_lo,
                     max(new_lo, _log_int(rng, 1, 128)), rng.choice((0.0, 0.0, 0.1, 0.5)), rng.choice((0.0, 0.0, 0.3)))
    dtype = rng.choice(("f16", "bf16", "f16", "bf16", "f32"))
    page = 1 << rng.randint(3, 8)
    order = rng.choice(("page", "token"))
    heads, kv = rng.choice(((32, 32), (32, 8), (32, 4), (28, 4), (12, 4), (4, 4), (4, 1), (5, 5)))
    hd = rng.choice((128, 128, 64))
    if u < 0.4:
        rows = _log_int(rng, 1, 8192)
        return _append(rows // 2 + 1 if dtype == "f32" else rows, heads, kv, hd, page, dtype, order, rng.random() < 0.8)
    while True:
        batch, new = _log_int(rng, 1, 64), rng.choice((1, _log_int(rng, 1, 2048), _log_int(rng, 1, 128)))
        hi = rng.choice((0, _log_int(rng, 1, 2000), _log_int(rng, 16, 131072)))
        lo = hi if rng.random() < 0.5 else hi // rng.randint(2, 8)
        window = rng.choice((0, 0, 0, _log_int(rng, 1, 4096)))
        mask = new <= 128 and rng.random() < 0.25
        c = _attn(batch, new, lo, hi, heads, kv, hd, page, dtype, order, window, mask)
        w = work(c)
        scores = 4.0 * batch * heads * new * (hi + new)
        if w["bytes"] < 5e8 and w["flops"] < (2e10 if dtype == "f32" else 1.5e11) and scores < 1.5e9 \
                and batch * (hi + new) * kv * hd < 1.5e8:
            return c


# ---- inputs ------------------------------------------------------------------------


def _pool(case, layers, n_pages, gen):
    """Pages of random keys or values as [layer][page][head][position][hd], in either order of memory."""
    kv, page, hd, dt = case["kv_heads"], case["page"], case["hd"], DTYPES[case["dtype"]]
    if case["order"] == "page":
        return torch.randn(layers, n_pages, kv, page, hd, device=DEV, generator=gen, dtype=dt)
    return torch.randn(layers, n_pages, page, kv, hd, device=DEV, generator=gen, dtype=dt).transpose(2, 3)


def _lengths(rng, lo, hi, n):
    return rng.integers(lo, hi + 1, size=n).astype(np.int64)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _plan_inputs(case, seed):
    rng = np.random.default_rng(seed)
    b, page = case["batch"], case["page"]
    ctx, new = _lengths(rng, case["lo"], case["hi"], b), _lengths(rng, case["new_lo"], case["new_hi"], b)
    held = -(-(ctx + rng.integers(0, page, size=b)) // page)  # the last step's block may reach into a further page
    ended = rng.random(b) < case["done"]
    ctx[ended], new[ended] = 0, 0
    width = -(-(case["hi"] + case["new_hi"] + page) // page)
    want = int(np.maximum(-(-(ctx + new) // page) - held, 0).sum())
    count = int(want * (1.0 - case["short"]))
    n_pages = b * width  # the other pages are somebody else's
    pages = rng.permutation(n_pages)
    table = np.full((b, width), -1, np.int64)
    table[np.arange(width)[None, :] < held[:, None]] = pages[:held.sum()]
    ring, head = rng.permutation(n_pages), int(rng.integers(0, n_pages))
    ring[(head + np.arange(count)) % n_pages] = pages[held.sum():held.sum() + count]
    rows = b * case["new_hi"]
    return dict(ctx=_i32(ctx), new=_i32(new), table=_i32(table), held=_i32(held), ring=_i32(ring),
                state=_i32([head, count, 0, 0]), page=page, rows=rows)


def _append_inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    t, h, kv, hd, page = case["rows"], case["heads"], case["kv_heads"], case["hd"], case["page"]
    n_pages = 2 * -(-t // page) + 1
    # one product gives q, k and v of a row side by side
    qkv = torch.randn(t, (h + 2 * kv) * hd, device=DEV, generator=gen, dtype=DTYPES[case["dtype"]])
    q, k, v = qkv[:, :h * hd].view(t, h, hd), qkv[:, h * hd:(h + kv) * hd].view(t, kv, hd), qkv[:, (h + kv) * hd:].view(t, kv, hd)
    pages = rng.permutation(n_pages)[:-(-t // page) + 1]
    start = int(rng.integers(0, page))
    at = start + np.arange(t)
    slots = torch.from_numpy(pages[at // page] * page + at % page).to(DEV)
    first = int(rng.integers(0, 4096))
    pos = _i32(first + np.arange(t))
    i = torch.arange(hd // 2, device=DEV, dtype=torch.float64)
    ang = torch.arange(first + t, device=DEV, dtype=torch.float64)[:, None] * 1e4 ** (-2.0 * i / hd)
    rope = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()  # [position][hd/2][2]
    return dict(q=q, k=k, v=v, slots=slots, pos=pos, rope=rope if case["rope"] else None,
                kp=_pool(case, 1, n_pages, gen), vp=_pool(case, 1, n_pages, gen))


def _attn_inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    b, n, h, hd, page = case["batch"], case["new"], case["heads"], case["hd"], case["page"]
    ctx = _lengths(rng, case["lo"], case["hi"], b)
    total = ctx + n
    used = -(-total // page)
    n_pages, width = int(used.sum()) + 3, -(-(case["hi"] + n) // page)
    pages = rng.permutation(n_pages)
    table = np.full((b, width), -1, np.int64)
    table[np.arange(width)[None, :] < used[:, None]] = pages[:used.sum()]
    q = 2.0 * torch.randn(b * n, h, hd, device=DEV, generator=gen)
    mask = None
    if case["mask"]:
        # a forest: every token sees itself and its ancestors (bit j of word j/32)
        parent = rng.integers(-1, np.arange(n), size=(b, n))
        see = np.zeros((b, n, n), bool)
        for i in range(n):
            p = parent[:, i]
            see[:, i] = np.where(p[:, None] >= 0, see[np.arange(b), np.maximum(p, 0)], False)
            see[:, i, i] = True
        words = -(-n // 32)
        bits = np.zeros((b * n, words), np.int64)
        for j in range(n):
            bits[:, j // 32] |= see[:, :, j].reshape(-1).astype(np.int64) << (j % 32)
        mask = torch.from_numpy(bits.astype(np.uint32).view(np.int32)).to(DEV)
    return dict(q=q.to(DTYPES[case["dtype"]]), kp=_pool(case, 1, n_pages, gen), vp=_pool(case, 1, n_pages, gen),
                table=_i32(table), row_start=_i32(np.arange(b + 1) * n), seq_len=_i32(total), mask=mask,
                window=case["window"], scale=hd ** -0.5, new=n, page=page)


INPUTS = {"plan": _plan_inputs, "append": _append_inputs, "attention": _attn_inputs}


def prepare(case, seed):
    s = dict(INPUTS[case["op"]](case, seed), op=case["op"])
    if s["op"] == "plan":
        b, dev = case["batch"], DEV
        s["out"] = dict(table=torch.empty_like(s["table"]), held=torch.empty_like(s["held"]), state=torch.zeros_like(s["state"]),
                        row_start=torch.empty(b + 1, dtype=torch.int32, device=dev), seq_len=torch.empty(b, dtype=torch.int32, device=dev),
                        granted=torch.empty(b, dtype=torch.int32, device=dev), slots=torch.empty(s["rows"], dtype=torch.int64, device=dev),
                        positions=torch.empty(s["rows"], dtype=torch.int32, device=dev))
    else:
        s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV)
        if s["op"] == "attention":
            s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
    if own:
        from paper_2403_00835_gb300 import paged
        if s["op"] == "plan":
            o = s["out"]
            s["tables"] = paged.PageTables(s["table"], s["held"], s["ring"], s["state"], s["page"])
            s["tables_out"] = paged.PageTables(o["table"], o["held"], s["ring"], o["state"], s["page"])
            s["plan_rows"] = paged.PageRows(o["row_start"], o["seq_len"], o["granted"], o["slots"], o["positions"])
        else:
            s["cache"] = paged.PagedCache(s["kp"], s["vp"], case["heads"])
            if s["op"] == "attention":
                s["plan_rows"] = paged.PageRows(s["row_start"], s["seq_len"])
                s["tables"] = paged.PageTables(s["table"], page_size=s["page"])
    return s


# ---- one pass ----------------------------------------------------------------------


def run(s):
    return (RUN_OWN if own else RUN_PLAIN)[s["op"]](s)


def _own_plan(s):
    from paper_2403_00835_gb300 import paged
    paged.plan(s["tables"], s["plan_rows"], s["ctx"], s["new"], out=s["tables_out"])
    return dict(s["out"], ring=s["ring"])


def _own_append(s):
    if s["rope"] is None:
        s["cache"].append(0, s["k"], s["v"], s["slots"])
        return {"k": s["kp"], "v": s["vp"]}
    s["cache"].append(0, s["k"], s["v"], s["slots"], q=s["q"], q_out=s["out"], rope=s["rope"], positions=s["pos"])
    return {"k": s["kp"], "v": s["vp"], "q": s["out"]}


def _own_attention(s):
    s["cache"].attention(0, s["q"], s["plan_rows"], s["tables"], out=s["out"], lse=s["lse"], scale=s["scale"],
                         window=s["window"], block_mask=s["mask"])
    return {"o": s["out"], "lse": s["lse"]}


def _plain_plan(s):
    ctx, new, held, table, ring, page = s["ctx"].long(), s["new"].long(), s["held"].long(), s["table"], s["ring"], s["page"]
    n, (b, width), dev = ring.numel(), table.shape, table.device
    head, count = s["state"][0].long(), s["state"][1].long()
    rows = new.clamp(min=0)
    end = rows.cumsum(0)
    valid = (ctx >= 0) & (new >= 0) & (ctx + new <= width * page) & (end <= s["rows"])
    need = torch.where(valid, (ctx + new + page - 1) // page, held)
    grow = (need - held).clamp(min=0)
    incl = grow.cumsum(0)
    granted = valid & ((grow == 0) | (incl <= count))
    held2 = torch.where(granted, need, held)
    j = torch.arange(width, device=dev)[None, :]
    fresh = ring[(head + (incl - grow)[:, None] + j - held[:, None]) % n]
    table2 = torch.where(j < torch.minimum(held, held2)[:, None], table, torch.where(j < held2[:, None], fresh, -1))
    shrink = (held - held2).clamp(min=0)
    back = shrink.cumsum(0) - shrink
    gone = (j >= held2[:, None]) & (j < held[:, None])
    # pages that stay are written to a place past the ring
    to = torch.where(gone, (head + count + back[:, None] + j - held2[:, None]) % n, n)
    more = torch.cat([ring, ring[:1]])
    more[to.reshape(-1)] = table.reshape(-1)
    ring.copy_(more[:n])
    taken = torch.where(granted, grow, 0).sum()
    state = torch.zeros_like(s["state"])
    state[0], state[1] = (head + taken) % n, count - taken + shrink.sum()
    t = torch.arange(s["rows"], device=dev)
    at = torch.searchsorted(end, t, right=True)
    live = at < b
    at = at.clamp(max=b - 1)
    live &= granted[at]
    pos = torch.where(live, ctx[at] + t - (end - rows)[at], 0)
    slots = torch.where(live, table2[at, (pos // page).clamp(max=width - 1)].long() * page + pos % page, -1)
    return {"table": table2, "held": held2.int(), "ring": ring, "state": state,
            "row_start": torch.cat([torch.zeros_like(end[:1]), end]).int(), "seq_len": torch.where(granted, ctx + new, 0).int(),
            "granted": granted.int(), "slots": slots, "positions": pos.int()}


def _rotate(x, cs):
    x = x.float()
    a, b = x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _plain_append(s):
    k, v, dt, page = s["k"], s["v"], s["k"].dtype, s["kp"].shape[3]
    out = {"k": s["kp"], "v": s["vp"]}
    if s["rope"] is not None:
        cs = s["rope"][s["pos"].long()]
        k = _rotate(k, cs).to(dt)
        out["q"] = _rotate(s["q"], cs).to(dt)
    p, i = s["slots"] // page, s["slots"] % page
    s["kp"][0].transpose(1, 2)[p, i] = k
    s["vp"][0].transpose(1, 2)[p, i] = v
    return out


def _visible(s, ctx, idx, keys, new_of_row):
    """[request][new token][key]: which keys a row sees."""
    j = keys[None, None, :] - ctx[:, None, None]
    if s["mask"] is not None:
        bits = s["mask"].long() & 0xFFFFFFFF
        jc = j.clamp(0, 32 * bits.shape[1] - 1)
        word = torch.gather(bits[new_of_row], 2, (jc // 32).expand(-1, idx.shape[1], -1))
        inside = (word >> (jc % 32)) & 1 == 1
    else:
        inside = keys[None, None, :] <= idx[:, :, None]
    seen = (j < 0) | (inside & (j < s["new"]))
    if s["window"]:
        seen = seen & (idx[:, :, None] - keys[None, None, :] < s["window"])
    return seen


def _plain_attention(s):
    q, table, page, n = s["q"], s["table"].long(), s["page"], s["new"]
    t, h, hd = q.shape
    b, width = table.shape
    kv = s["kp"].shape[2]
    ctx = s["seq_len"].long() - n
    rows = s["row_start"][:-1].long()[:, None] + torch.arange(n, device=q.device)[None, :]
    idx = ctx[:, None] + torch.arange(n, device=q.device)[None, :]
    keys = torch.arange(width * page, device=q.device)
    seen = _visible(s, ctx, idx, keys, rows)[:, None, None]
    at = table.clamp(min=0)
    k = s["kp"][0][at].transpose(1, 2).reshape(b, kv, 1, width * page, hd).float()
    v = s["vp"][0][at].transpose(1, 2).reshape(b, kv, 1, width * page, hd).float()
    qg = q[rows].float().view(b, n, kv, h // kv, hd).permute(0, 2, 3, 1, 4)
    sc = (qg @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = sc.sub_(top.clamp(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / total.clamp(min=1e-30)
    lse = (top + total.log()).squeeze(-1)
    return {"o": o.permute(0, 3, 1, 2, 4).reshape(t, h, hd).to(q.dtype), "lse": lse.permute(0, 3, 1, 2).reshape(t, h)}


RUN_OWN = {"plan": _own_plan, "append": _own_append, "attention": _own_attention}
RUN_PLAIN = {"plan": _plain_plan, "append": _plain_append, "attention": _plain_attention}


# ---- what a pass cannot do without ---------------------------------------------------


def work(case):
    if case["op"] == "plan":
        b, page = case["batch"], case["page"]
        width = -(-(case["hi"] + case["new_hi"] + page) // page)
        mean = (1 - case["done"]) * (case["lo"] + case["hi"]) / 2 / page
        # lengths and held pages in; the held part of the tables in, whole tables, rows and per-request results out
        return {"bytes": b * (12 + 4 * mean + 4 * width + 16) + 12 * b * case["new_hi"], "flops": 0}
    es, hd = (4 if case["dtype"] == "f32" else 2), case["hd"]
    if case["op"] == "append":
        t, kv, h = case["rows"], case["kv_heads"], case["heads"] if case["rope"] else 0
        return {"bytes": 2 * es * t * hd * (h + 2 * kv) + t * (12 + (4 * hd if case["rope"] else 0)),
                "flops": 3.0 * t * hd * (h + kv) if case["rope"] else 0}
    b, n, h, kv, w = case["batch"], case["new"], case["heads"], case["kv_heads"], case["window"]
    mean = (case["lo"] + case["hi"]) / 2
    seen = mean + (n + 1) / 2
    keys = mean + n
    if w:
        seen, keys = min(seen, w), min(keys, w + n)
    return {"bytes": es * (2 * b * n * h * hd + 2 * b * kv * hd * keys) + 4 * b * n * h + 4 * b * keys / case["page"],
            "flops": 4.0 * hd * h * b * n * seen}


# ---- the same in 64 bits -------------------------------------------------------------


def exact(case, seed):
    if case["op"] == "plan":
        return None  # whole numbers
    s = INPUTS[case["op"]](case, seed)
    if case["op"] == "append":
        out = {}
        hd, page = case["hd"], case["page"]
        ang = None
        if case["rope"]:
            cs = s["rope"].double()[s["pos"].long()]
            ang = torch.complex(cs[..., 0], cs[..., 1])[:, None, :]

        def turn(x):
            if ang is None:
                return x.double()
            z = torch.complex(x[..., :hd // 2].double(), x[..., hd // 2:].double()) * ang
            return torch.cat([z.real, z.imag], -1)

        for name, x, pool in (("k", turn(s["k"]), s["kp"]), ("v", s["v"].double(), s["vp"])):
            flat = pool.double()
            for t0 in range(0, case["kv_heads"]):
                one = flat[0, :, t0].reshape(-1, hd)
                one[s["slots"]] = x[:, t0]
                flat[0, :, t0] = one.view(-1, page, hd)
            out[name] = flat
        if case["rope"]:
            out["q"] = turn(s["q"])
        return out
    t, h, hd = s["q"].shape
    n, group = case["new"], case["heads"] // case["kv_heads"]
    o = torch.zeros(t, h, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((t, h), -math.inf, dtype=torch.float64, device=DEV)
    for b, total in enumerate(s["seq_len"].tolist()):
        ctx, r0 = total - n, b * n
        pages = s["table"][b, :-(-total // case["page"])].long()
        for g in range(case["kv_heads"]):
            k = s["kp"][0, pages, g].reshape(-1, hd)[:total].double()
            v = s["vp"][0, pages, g].reshape(-1, hd)[:total].double()
            for i0 in range(0, n, 256):
                i = torch.arange(i0, min(n, i0 + 256), device=DEV)
                at = torch.arange(total, device=DEV)
                if s["mask"] is not None:
                    see = torch.ones(len(i), total, dtype=torch.bool, device=DEV)
                    j = torch.arange(n, device=DEV)
                    see[:, ctx:] = (s["mask"][r0 + i][:, j // 32].long() >> (j % 32)) & 1 > 0
                else:
                    see = at[None, :] <= ctx + i[:, None]
                if case["window"]:
                    see &= at[None, :] > ctx + i[:, None] - case["window"]
                for hh in range(g * group, (g + 1) * group):
                    sc = (s["q"][r0 + i, hh].double() @ k.T * s["scale"]).masked_fill(~see, -math.inf)
                    l = torch.logsumexp(sc, -1)
                    p = torch.where(see, (sc - l.clamp(min=-1e300)[:, None]).exp(), 0.0)
                    o[r0 + i, hh], lse[r0 + i, hh] = p @ v, l
    return {"o": o, "lse": lse}
