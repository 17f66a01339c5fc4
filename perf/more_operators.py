"""Performance cases of what a sampled decode over long streams adds to the paged
key/value cache: rotary tables from scaled frequencies (``paged.rope_table``), the write of
keys with norms of queries and keys per head and a rotation of part of the head
(``PagedCache.append``), attention within a window plus the first tokens
(``PagedCache.attention`` with ``sinks``), and the verification of drafted tokens against the
target's probabilities (``verify.DraftVerifier``).

``own`` false computes the same with elementary torch operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rope(positions, dims, theta, factor, name=None):
    """A table of all positions; the low frequencies are divided by `factor`."""
    c = dict(op="rope", positions=positions, dims=dims, theta=theta, factor=factor)
    return dict(c, name=name) if name else c


def _append(rows, heads, kv_heads, hd, page, dtype, order, dims, pairs, norms="qk", name=None):
    """order: "page" has a page's tokens of one head together, "token" one token's heads.
    dims: how many of a head's first values are rotated (0: none); pairs: "half" or
    "interleaved"; norms: of the queries ("q"), of the keys ("k"), both or none."""
    c = dict(op="append", rows=rows, heads=heads, kv_heads=kv_heads, hd=hd, page=page, dtype=dtype, order=order,
             dims=dims, pairs=pairs, norms=norms)
    return dict(c, name=name) if name else c


def _attn(batch, new, lo, hi, heads, kv_heads, hd, page, dtype, window, sinks, order="page", mask=False, name=None):
    """`new` tokens for each request after lo..hi ones, of which the first `sinks` and
    those within `window` are seen; the pages between are gone."""
    c = dict(op="attention", batch=batch, new=new, lo=lo, hi=hi, heads=heads, kv_heads=kv_heads, hd=hd, page=page,
             dtype=dtype, window=window, sinks=sinks, order=order, mask=mask)
    return dict(c, name=name) if name else c


def _verify(batch, lo, hi, vocab, dtype, probs=False, heat="one", name=None):
    """lo..hi rows a request (its head and the drafts after it); probs: the drafts come with
    their distributions, else they are certain (a Jacobi block, an n-gram); heat: the
    temperature is one, or each request has its own, some of them none (greedy)."""
    c = dict(op="verify", batch=batch, lo=lo, hi=hi, vocab=vocab, dtype=dtype, probs=probs, heat=heat)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a server stretches a small decoder's positions
        _rope(8192, 64, 1e4, 4.0, name="rope_8192"),
        # the table of a very long context, made once when a model is loaded
        _rope(1 << 20, 128, 1e6, 32.0, name="rope_1m"),
        # one user's block of 16: launch latency
        _append(16, 32, 8, 128, 16, "f16", "page", 128, "half", name="append_block16"),
        # a batch of blocks; half of each head is rotated, neighbours in pairs; token-major pages
        _append(256, 32, 8, 128, 64, "bf16", "token", 64, "interleaved", name="append_batch256"),
        # a chunk of prompts
        _append(8192, 32, 32, 128, 64, "bf16", "page", 128, "half", name="append_prefill8192"),
        # the small fp32 decoder's block of 8, some way into a stream
        _attn(1, 8, 200, 400, 4, 4, 64, 16, "f32", 64, 4, name="attn_tiny_f32_n8"),
        # greedy decoding of a full batch of long streams: one token a request
        _attn(64, 1, 8000, 60000, 32, 8, 128, 64, "bf16", 4096, 4, name="attn_stream_batch64"),
        # blocks of 16 of eight streams
        _attn(8, 16, 3000, 20000, 32, 32, 128, 32, "f16", 1024, 64, "token", name="attn_block16_batch8"),
        # a chunk of a long prompt
        _attn(1, 2048, 4096, 4096, 32, 32, 128, 64, "bf16", 1024, 4, name="attn_chunk2048"),
        # one user's Jacobi block, fp32 logits
        _verify(1, 16, 16, 32000, "f32", name="verify_block16"),
        # a batch with a draft model's distributions, each request with its temperature
        _verify(32, 5, 9, 32256, "bf16", True, "own", name="verify_batch32_probs"),
        # a full server's drafts over a large vocabulary
        _verify(128, 4, 8, 131072, "bf16", False, "own", name="verify_batch128"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = ((32, 32), (32, 8), (32, 4), (28, 4), (12, 4), (4, 4), (4, 1), (5, 5))


def draw(rng):
    u = rng.random()
    if u < 0.1:
        return _rope(_log_int(rng, 1, 1 << 20), 16 * rng.randint(1, 8), rng.choice((1e4, 1e5, 1e6)), rng.choice((1.0, 4.0, 32.0)))
    dtype = rng.choice(("f16", "bf16", "f16", "bf16", "f32"))
    page = 1 << rng.randint(3, 8)
    order = rng.choice(("page", "token"))
    heads, kv = rng.choice(HEADS)
    hd = rng.choice((128, 128, 64))
    if u < 0.4:
        rows = _log_int(rng, 1, 8192)
        dims = rng.choice((hd, hd, hd // 2, hd // 4, 16 * rng.randint(1, hd // 16), 0))
        norms = rng.choice(("qk", "qk", "qk", "q", "k", ""))
        if dims == 0 and not norms:
            norms = "k"
        return _append(rows // 2 + 1 if dtype == "f32" else rows, heads, kv, hd, page, dtype, order, dims,
                       rng.choice(("half", "interleaved")), norms)
    if u < 0.7:
        while True:
            batch, new = _log_int(rng, 1, 64), rng.choice((1, _log_int(rng, 1, 2048), _log_int(rng, 1, 128)))
            hi = rng.choice((0, _log_int(rng, 1, 2000), _log_int(rng, 16, 131072)))
            lo = hi if rng.random() < 0.5 else hi // rng.randint(2, 8)
            window, sinks = _log_int(rng, 1, 4096), rng.choice((4, _log_int(rng, 1, 300)))
            mask = new <= 128 and rng.random() < 0.2
            c = _attn(batch, new, lo, hi, heads, kv, hd, page, dtype, window, sinks, order, mask)
            w = work(c)
            keys = sinks + window + new
            if w["bytes"] < 6e8 and w["flops"] < (1e10 if dtype == "f32" else 4e10) \
                    and 4.0 * batch * heads * new * keys < 2e9 and batch * keys * heads * hd < 1.2e9:
                return c
    while True:
        batch, lo = _log_int(rng, 1, 128), _log_int(rng, 1, 16)
        c = _verify(batch, lo, lo + rng.choice((0, _log_int(rng, 1, 16))), _log_int(rng, 500, 160000),
                    rng.choice(("f32", "bf16", "f16")), rng.random() < 0.4, rng.choice(("one", "own", "own")))
        if work(c)["bytes"] < 2.2e8 and c["batch"] * c["hi"] * c["vocab"] < 1.3e8:
            return c


# ---- inputs ------------------------------------------------------------------------


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _frequencies(case):
    """Divided by the factor where a turn takes over 4096 positions, kept where it takes under 128."""
    out = []
    for i in range(case["dims"] // 2):
        f = case["theta"] ** (-2.0 * i / case["dims"])
        keep = min(1.0, max(0.0, (math.log(4096) - math.log(2 * math.pi / f)) / math.log(32)))
        out.append(f * keep + f / case["factor"] * (1.0 - keep))
    return out


def _rope_inputs(case, seed):
    # (another seed: another base, as another model has)
    case = dict(case, theta=case["theta"] * (1.0 + 0.01 * (seed % 89)))
    return dict(freq=_frequencies(case), amp=0.1 * math.log(case["factor"]) + 1.0, n=case["positions"])


def _pool(case, n_pages, gen):
    """Pages of random keys or values as [1][page][head][position][hd], in either order of memory."""
    kv, page, hd, dt = case["kv_heads"], case["page"], case["hd"], DTYPES[case["dtype"]]
    if case["order"] == "page":
        return torch.randn(1, n_pages, kv, page, hd, device=DEV, generator=gen, dtype=dt)
    return torch.randn(1, n_pages, page, kv, hd, device=DEV, generator=gen, dtype=dt).transpose(2, 3)


def _append_inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    t, h, kv, hd, page, dims = case["rows"], case["heads"], case["kv_heads"], case["hd"], case["page"], case["dims"]
    dt = DTYPES[case["dtype"]]
    n_pages = 2 * -(-t // page) + 1
    # one product gives q, k and v of a row side by side
    qkv = torch.randn(t, (h + 2 * kv) * hd, device=DEV, generator=gen)
    qkv = (qkv * (0.5 + 2.0 * torch.rand(t, 1, device=DEV, generator=gen))).to(dt)
    q, k, v = qkv[:, :h * hd].view(t, h, hd), qkv[:, h * hd:(h + kv) * hd].view(t, kv, hd), qkv[:, (h + kv) * hd:].view(t, kv, hd)
    pages = rng.permutation(n_pages)[:-(-t // page) + 1]
    at = int(rng.integers(0, page)) + np.arange(t)
    slots = torch.from_numpy(pages[at // page] * page + at % page).to(DEV)
    first = int(rng.integers(0, 4096))
    rope = None
    if dims:
        i = torch.arange(dims // 2, device=DEV, dtype=torch.float64)
        ang = torch.arange(first + t, device=DEV, dtype=torch.float64)[:, None] * 1e4 ** (-2.0 * i / dims)
        rope = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()  # [position][dims/2][2]
    gains = {n: (1.0 + 0.2 * torch.randn(hd, device=DEV, generator=gen)).to(dt) for n in "qk"}
    return dict(q=q, k=k, v=v, slots=slots, pos=_i32(first + np.arange(t)), rope=rope, pairs=case["pairs"],
                qn=gains["q"] if "q" in case["norms"] else None, kn=gains["k"] if "k" in case["norms"] else None,
                eps=1e-6, kp=_pool(case, n_pages, gen), vp=_pool(case, n_pages, gen))


def _attn_inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    b, n, h, hd, page = case["batch"], case["new"], case["heads"], case["hd"], case["page"]
    total = rng.integers(case["lo"], case["hi"] + 1, size=b).astype(np.int64) + n
    width = -(-(case["hi"] + n) // page)
    # the pages of the first tokens and from the oldest row's window on; the ones between are gone
    j = np.arange(width)[None, :]
    keep = (j * page < case["sinks"]) | ((j + 1) * page > (total - n - case["window"] + 1)[:, None])
    keep &= j * page < total[:, None]
    n_pages = int(keep.sum()) + 3
    table = np.full((b, width), -1, np.int64)
    table[keep] = rng.permutation(n_pages)[:keep.sum()]
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
        bits = np.zeros((b * n, -(-n // 32)), np.int64)
        for i in range(n):
            bits[:, i // 32] |= see[:, :, i].reshape(-1).astype(np.int64) << (i % 32)
        mask = torch.from_numpy(bits.astype(np.uint32).view(np.int32)).to(DEV)
    return dict(q=q.to(DTYPES[case["dtype"]]), kp=_pool(case, n_pages, gen), vp=_pool(case, n_pages, gen),
                table=_i32(table), row_start=_i32(np.arange(b + 1) * n), seq_len=_i32(total), mask=mask,
                window=case["window"], sinks=case["sinks"], scale=hd ** -0.5, new=n, page=page)


def _verify_inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    b, vocab = case["batch"], case["vocab"]
    n = rng.permutation(case["lo"] + np.arange(b) % (case["hi"] - case["lo"] + 1))
    start = np.concatenate([[0], np.cumsum(n)])
    t = int(start[-1])
    # each row has a favourite of 0.2 to 0.9 or so, and the drafts name it often
    z = 2.0 * torch.randn(t, vocab, device=DEV, generator=gen)
    best = torch.randint(0, vocab, (t,), device=DEV, generator=gen)
    z[torch.arange(t, device=DEV), best] = math.log(vocab) + 2.0 + 4.0 * torch.rand(t, device=DEV, generator=gen) - 1.0
    heat = np.ones(b)
    if case["heat"] == "own":
        heat = np.where(rng.random(b) < 0.2, 0.0, rng.uniform(0.5, 1.3, size=b))
    heat = torch.from_numpy(heat.astype(np.float32)).to(DEV)
    probs = None
    if case["probs"]:
        # the draft model is near the target; drafts are drawn from it
        probs = torch.softmax(z + 0.5 * torch.randn(t, vocab, device=DEV, generator=gen), -1)
        follow = (probs / torch.empty_like(probs).exponential_(generator=gen)).argmax(-1)
    else:
        other = torch.randint(0, vocab, (t,), device=DEV, generator=gen)
        follow = torch.where(torch.rand(t, device=DEV, generator=gen) < 0.8, best, other)
    tokens = torch.randint(0, vocab, (t,), device=DEV, generator=gen)
    tokens[1:] = follow[:-1]  # (the token after row i is row i + 1's; a request's first is its head)
    race = torch.empty(b, vocab, device=DEV).exponential_(generator=gen).clamp_(min=1e-30)
    return dict(z=z.to(DTYPES[case["dtype"]]), tokens=tokens.int(), row_start=_i32(start), seq_len=_i32(n + 100),
                u=torch.rand(t, device=DEV, generator=gen), race=race, heat=heat if case["heat"] == "own" else None, probs=probs)


INPUTS = {"rope": _rope_inputs, "append": _append_inputs, "attention": _attn_inputs, "verify": _verify_inputs}


def prepare(case, seed):
    s = dict(INPUTS[case["op"]](case, seed), op=case["op"])
    if s["op"] == "rope":
        s["out"] = torch.empty(s["n"], len(s["freq"]), 2, device=DEV)
    elif s["op"] == "verify":
        s["out"] = [torch.empty(case["batch"], dtype=torch.int32, device=DEV) for _ in range(2)]
        s["p"] = torch.zeros(s["z"].shape[0], device=DEV)
    else:
        s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV)
        if s["op"] == "attention":
            s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
    if own:
        from paper_2403_00835_gb300 import paged, verify
        if s["op"] in ("append", "attention"):
            s["cache"] = paged.PagedCache(s["kp"], s["vp"], case["heads"])
        if s["op"] in ("verify", "attention"):
            s["plan_rows"] = paged.PageRows(s["row_start"], s["seq_len"])
        if s["op"] == "attention":
            s["tables"] = paged.PageTables(s["table"], page_size=s["page"])
        if s["op"] == "verify":
            s["verifier"] = verify.DraftVerifier(max_rows=s["z"].shape[0], max_batch=case["batch"])
    return s


# ---- one pass ----------------------------------------------------------------------


def run(s):
    return (RUN_OWN if own else RUN_PLAIN)[s["op"]](s)


def _own_rope(s):
    from paper_2403_00835_gb300 import paged
    return paged.rope_table(s["n"], s["freq"], amplitude=s["amp"], out=s["out"])


def _own_append(s):
    s["cache"].append(0, s["k"], s["v"], s["slots"], q=s["q"], q_out=s["out"], rope=s["rope"],
                      positions=None if s["rope"] is None else s["pos"], q_norm=s["qn"], k_norm=s["kn"], eps=s["eps"],
                      interleaved=s["pairs"] == "interleaved")
    return {"k": s["kp"], "v": s["vp"], "q": s["out"]}


def _own_attention(s):
    s["cache"].attention(0, s["q"], s["plan_rows"], s["tables"], out=s["out"], lse=s["lse"], scale=s["scale"],
                         window=s["window"], sinks=s["sinks"], block_mask=s["mask"])
    return {"o": s["out"], "lse": s["lse"]}


def _own_verify(s):
    s["verifier"].verify(s["z"], s["tokens"], s["plan_rows"], uniforms=s["u"], race=s["race"], temperature=s["heat"],
                         draft_probs=s["probs"], accepted=s["out"][0], next_tokens=s["out"][1], target_probs=s["p"])
    return {"accepted": s["out"][0], "next": s["out"][1], "p": s["p"]}


def _plain_rope(s):
    f = torch.tensor(s["freq"], dtype=torch.float64).to(DEV, non_blocking=True)
    ang = torch.arange(s["n"], device=DEV, dtype=torch.float64)[:, None] * f
    return torch.stack([ang.cos().mul_(s["amp"]), ang.sin().mul_(s["amp"])], -1).float()


def _normed(x, gain, eps):
    x = x.float()
    return x if gain is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * gain.float()


def _rotate(x, cs, pairs):
    if cs is None:
        return x
    r = 2 * cs.shape[1]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    if pairs == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_append(s):
    dt, page = s["k"].dtype, s["kp"].shape[3]
    cs = None if s["rope"] is None else s["rope"][s["pos"].long()]
    p, i = s["slots"] // page, s["slots"] % page
    s["kp"][0].transpose(1, 2)[p, i] = _rotate(_normed(s["k"], s["kn"], s["eps"]), cs, s["pairs"]).to(dt)
    s["vp"][0].transpose(1, 2)[p, i] = s["v"]
    return {"k": s["kp"], "v": s["vp"], "q": _rotate(_normed(s["q"], s["qn"], s["eps"]), cs, s["pairs"]).to(dt)}


def _plain_attention(s):
    q, table, page, n, sinks, window = s["q"], s["table"].long(), s["page"], s["new"], s["sinks"], s["window"]
    t, h, hd = q.shape
    b, width = table.shape
    kv, dev = s["kp"].shape[2], q.device
    total = s["seq_len"].long()
    # the keys that some row of a request may see: the first ones, then those from its oldest row's window on
    near = window + n - 1
    first = (total - near).clamp(min=0)[:, None]
    head = torch.arange(sinks, device=dev)[None, :].expand(b, -1)
    pos = torch.cat([head, first + torch.arange(near, device=dev)[None, :]], 1)  # [request][key]
    real = torch.cat([head < first, pos[:, sinks:] < total[:, None]], 1)
    idx = total[:, None] - n + torch.arange(n, device=dev)[None, :]  # [request][row]
    rows = s["row_start"][:-1].long()[:, None] + torch.arange(n, device=dev)[None, :]
    gap = idx[:, :, None] - pos[:, None, :]
    seen = real[:, None, :] & ((gap < window) | (pos < sinks)[:, None, :])
    if s["mask"] is None:
        seen = seen & (gap >= 0)
    else:
        j = pos - (total - n)[:, None]
        bits = (s["mask"].long() & 0xFFFFFFFF)[rows]
        word = torch.gather(bits, 2, (j.clamp(0, n - 1) // 32)[:, None, :].expand(-1, n, -1))
        seen = seen & ((j < 0)[:, None, :] | ((word >> (j.clamp(min=0) % 32)[:, None, :]) & 1 == 1))
    seen = seen[:, None, None]
    at = pos.clamp(max=width * page - 1)
    page_no, off = torch.gather(table, 1, at // page).clamp(min=0), at % page
    k = s["kp"][0][page_no, :, off].float().transpose(1, 2)[:, :, None]  # [request][kv head][1][key][hd]
    v = s["vp"][0][page_no, :, off].float().transpose(1, 2)[:, :, None]
    qg = q[rows].float().view(b, n, kv, h // kv, hd).permute(0, 2, 3, 1, 4)
    sc = (qg @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = sc.sub_(top.clamp(min=-3e38)).exp_()
    sums = p.sum(-1, keepdim=True)
    o = (p @ v) / sums.clamp(min=1e-30)
    lse = (top + sums.log()).squeeze(-1)
    return {"o": o.permute(0, 3, 1, 2, 4).reshape(t, h, hd).to(q.dtype), "lse": lse.permute(0, 3, 1, 2).reshape(t, h)}


def _first_max(x):
    """The lowest index of each row's largest value."""
    at = torch.arange(x.shape[1], device=x.device)
    return torch.where(x == x.amax(-1, keepdim=True), at, x.shape[1]).amin(-1)


def _plain_verify(s):
    # in 64 bits: an acceptance and a race's winner are decided at borders
    t, vocab = s["z"].shape
    start = s["row_start"].long()
    b, dev = start.numel() - 1, start.device
    at = torch.arange(t, device=dev)
    req = torch.searchsorted(start[1:], at, right=True)
    last = at + 1 == start[1:][req]
    heat = torch.ones(b, dtype=torch.float64, device=dev) if s["heat"] is None else s["heat"].double()
    greedy = heat == 0
    z = s["z"].double()
    p = z / torch.where(greedy, 1.0, heat)[req][:, None]
    p = (p - p.amax(-1, keepdim=True)).exp_()
    p /= p.sum(-1, keepdim=True)
    draft = torch.cat([s["tokens"][1:], s["tokens"][:1]]).long()
    q = torch.ones(t, dtype=torch.float64, device=dev) if s["probs"] is None else s["probs"][at, draft].double()
    top = _first_max(s["z"])
    # (without a temperature the target's distribution is its favourite; the last row has no draft)
    pd = torch.where(last, 0.0, torch.where(greedy[req], (top == draft).double(), p[at, draft]))
    ok = torch.where(greedy[req], top == draft, s["u"].double() * q < pd) & ~last
    stop = torch.full((b,), t, device=dev).scatter_reduce(0, req, torch.where(ok, t, at), "amin")  # the row that decides
    ends = last[stop]
    w = p[stop]
    if s["probs"] is None:
        rest = w.scatter(1, draft[stop][:, None], 0.0)
    else:
        rest = (w - s["probs"][stop].double()).clamp(min=0.0)
    rest = torch.where((rest.amax(-1) > 0)[:, None], rest, w)
    drawn = _first_max(torch.where(ends[:, None], w, rest) / s["race"].double())
    return {"accepted": (stop - start[:-1] + 1).int(), "next": torch.where(greedy, top[stop], drawn).int(), "p": pd.float()}


RUN_OWN = {"rope": _own_rope, "append": _own_append, "attention": _own_attention, "verify": _own_verify}
RUN_PLAIN = {"rope": _plain_rope, "append": _plain_append, "attention": _plain_attention, "verify": _plain_verify}


# ---- what a pass cannot do without ---------------------------------------------------


def work(case):
    if case["op"] == "rope":
        return {"bytes": 4.0 * case["positions"] * case["dims"], "flops": 0}
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "append":
        t, kv, h, hd, dims = case["rows"], case["kv_heads"], case["heads"], case["hd"], case["dims"]
        normed = h * ("q" in case["norms"]) + kv * ("k" in case["norms"])
        return {"bytes": 2 * es * t * hd * (h + 2 * kv) + t * (12 + 4 * dims),
                "flops": 3.0 * t * dims * (h + kv) + 4.0 * t * hd * normed}
    if case["op"] == "verify":
        b, vocab = case["batch"], case["vocab"]
        rows = sum(case["lo"] + i % (case["hi"] - case["lo"] + 1) for i in range(b))
        # the logits once, the race, and of the drafts' distributions the row that decides
        drawn = 0.8 * b if case["heat"] == "own" else b
        return {"bytes": es * rows * vocab + 4.0 * drawn * vocab * (2 if case["probs"] else 1) + 12.0 * rows + 8.0 * b, "flops": 0}
    b, n, h, kv, hd, w, s = (case[k] for k in ("batch", "new", "heads", "kv_heads", "hd", "window", "sinks"))
    mean = (case["lo"] + case["hi"]) / 2
    seen = min(mean + (n + 1) / 2, w + s)
    keys = min(mean + n, s + w + n - 1)
    return {"bytes": es * (2 * b * n * h * hd + 2 * b * kv * hd * keys) + 4 * b * n * h + 4 * b * keys / case["page"],
            "flops": 4.0 * hd * h * b * n * seen}


# ---- the same in 64 bits -------------------------------------------------------------


def exact(case, seed):
    s = INPUTS[case["op"]](case, seed)
    if case["op"] == "verify":
        p = torch.zeros(s["z"].shape[0], dtype=torch.float64, device=DEV)
        heats = [1.0] * case["batch"] if s["heat"] is None else s["heat"].tolist()
        start = s["row_start"].tolist()
        for heat, r0, r1 in zip(heats, start, start[1:]):
            if r1 - r0 < 2:
                continue
            z, x = s["z"][r0:r1 - 1].double(), s["tokens"][r0 + 1:r1].long()[:, None]
            if heat == 0.0:
                top = s["z"][r0:r1 - 1].float().cpu().numpy().argmax(-1)  # (the first of equal ones)
                p[r0:r1 - 1] = (torch.from_numpy(top).to(DEV) == x.squeeze(1)).double()
            else:
                p[r0:r1 - 1] = (torch.gather(z, 1, x).squeeze(1) / heat - torch.logsumexp(z / heat, -1)).exp()
        return {"accepted": None, "next": None, "p": p}  # (whole numbers)
    if case["op"] == "rope":
        out = torch.empty(s["n"], len(s["freq"]), 2, device=DEV, dtype=torch.float64)
        pos = torch.arange(s["n"], device=DEV, dtype=torch.float64)
        amp = torch.full_like(pos, s["amp"])
        for i, f in enumerate(s["freq"]):
            out[:, i] = torch.view_as_real(torch.polar(amp, pos * f))
        return out
    if case["op"] == "append":
        hd, page, dims = case["hd"], case["page"], case["dims"]

        def done(x, gain):
            x = x.double()
            if gain is not None:
                x = x / (x.square().sum(-1, keepdim=True) / hd + s["eps"]).sqrt() * gain.double()
            if dims == 0:
                return x
            cs = s["rope"].double()[s["pos"].long()]
            turn = torch.complex(cs[..., 0], cs[..., 1])[:, None, :]
            y = x.clone()
            one, two = (slice(0, dims // 2), slice(dims // 2, dims)) if case["pairs"] == "half" else (slice(0, dims, 2), slice(1, dims, 2))
            z = torch.complex(x[..., one], x[..., two]) * turn
            y[..., one], y[..., two] = z.real, z.imag
            return y

        out = {}
        for name, x, pool in (("k", done(s["k"], s["kn"]), s["kp"]), ("v", s["v"].double(), s["vp"])):
            flat = pool.double()
            for g in range(case["kv_heads"]):
                one = flat[0, :, g].reshape(-1, hd)
                one[s["slots"]] = x[:, g]
                flat[0, :, g] = one.view(-1, page, hd)
            out[name] = flat
        out["q"] = done(s["q"], s["qn"])
        return out
    t, h, hd = s["q"].shape
    n, page, group = case["new"], case["page"], case["heads"] // case["kv_heads"]
    o = torch.zeros(t, h, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((t, h), -math.inf, dtype=torch.float64, device=DEV)
    for b, total in enumerate(s["seq_len"].tolist()):
        ctx, r0 = total - n, b * n
        for i0 in range(0, n, 256):
            i = torch.arange(i0, min(n, i0 + 256), device=DEV)
            oldest = max(0, ctx + i0 - case["window"] + 1)
            at = torch.cat([torch.arange(min(case["sinks"], oldest)), torch.arange(oldest, total)]).to(DEV)
            if s["mask"] is not None:
                new = at - ctx
                bit = (s["mask"][r0 + i][:, new.clamp(min=0) // 32].long() >> (new.clamp(min=0) % 32)) & 1 > 0
                see = (new < 0)[None, :] | bit
            else:
                see = at[None, :] <= ctx + i[:, None]
            see = see & ((at[None, :] > ctx + i[:, None] - case["window"]) | (at < case["sinks"])[None, :])
            pages, off = s["table"][b].long()[at // page], at % page
            for g in range(case["kv_heads"]):
                k, v = s["kp"][0, pages, g, off].double(), s["vp"][0, pages, g, off].double()
                for hh in range(g * group, (g + 1) * group):
                    sc = (s["q"][r0 + i, hh].double() @ k.T * s["scale"]).masked_fill(~see, -math.inf)
                    l = torch.logsumexp(sc, -1)
                    p = torch.where(see, (sc - l.clamp(min=-1e300)[:, None]).exp(), 0.0)
                    o[r0 + i, hh], lse[r0 + i, hh] = p @ v, l
    return {"o": o, "lse": lse}
