"""The model-step operators' workloads, for timing and for comparing outputs.

The operators are what a Call's model step does to the tokens of a ready batch
beside a paged key/value cache whose page lists and token ranges are lineage
arrays (sequence -> pages, sequence -> new tokens):

  rotary   rotary positions with several axes, forward and gradient
  append   rotary on q and k, then k and v into the cache's pages
  attend   a chunk of new tokens (or a single one) over the paged cache, heads
           sharing keys, optionally a sliding window with first tokens that
           stay visible
  weigh    the attention weight each cached token gathered
  evict    keep the heaviest tokens of each head, moved to fresh pages

`prepare` makes inputs from the seed alone: normal values, keys and queries
with a common direction on each sequence's first tokens (they draw weight, as
first tokens do), pages in random order, slots past a sequence's length
holding another sequence's old values, scores with a long tail and exact ties.
Sequence lengths belong to the case (`mix`), not to the seed.
"""
import functools
import math

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # a few frames' image tokens on their way back through a small tower: gradient, pairs side by side
        {"name": "rotary_grad_small", "op": "rotary", "tokens": 577, "heads": 12, "dim": 80, "dtype": "f32",
         "axes": 2, "interleaved": True, "inverse": True, "span": 64},
        # video tokens of a training batch: time, height and width
        {"name": "rotary_video", "op": "rotary", "tokens": 65_536, "heads": 32, "dim": 128, "dtype": "bf16",
         "axes": 3, "interleaved": False, "inverse": False, "span": 4096},
        # one new token for each sequence of a ready batch of 256
        {"name": "append_single", "op": "append", "seqs": 256, "new": 1, "len": 1000, "ragged": True, "mix": 1,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "axes": 1, "span": 1000},
        # prompts of documents' pages, ragged, arriving together
        {"name": "append_chunks", "op": "append", "seqs": 24, "new": 2048, "len": 4096, "ragged": True, "mix": 2,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "axes": 3, "span": 4096},
        # one user, one token: latency
        {"name": "attend_one", "op": "attend", "seqs": 1, "new": 1, "len": 777, "ragged": False, "mix": 3,
         "heads": 16, "kv_heads": 4, "dim": 64, "page": 16, "dtype": "f16", "window": 0, "sinks": 0},
        # single tokens of a ready batch, caches of 1 to 32 thousand tokens
        {"name": "attend_singles", "op": "attend", "seqs": 64, "new": 1, "len": 32_000, "ragged": True, "mix": 4,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "window": 0, "sinks": 0},
        # chunks of long prompts over what is cached already
        {"name": "attend_chunks", "op": "attend", "seqs": 8, "new": 2048, "len": 16_384, "ragged": True, "mix": 5,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "window": 0, "sinks": 0},
        # a stream of frames: a chunk of image tokens sees a window and the first tokens
        {"name": "attend_stream", "op": "attend", "seqs": 4, "new": 729, "len": 100_000, "ragged": True, "mix": 6,
         "heads": 28, "kv_heads": 4, "dim": 128, "page": 128, "dtype": "bf16", "window": 4096, "sinks": 4},
        # weight gathered while single tokens are generated
        {"name": "weigh_singles", "op": "weigh", "seqs": 32, "new": 1, "len": 16_000, "ragged": True, "mix": 7,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "window": 0, "sinks": 0,
         "decay": 1.0},
        # weight that a chunk's tokens give to what is cached
        {"name": "weigh_chunks", "op": "weigh", "seqs": 6, "new": 1024, "len": 16_384, "ragged": True, "mix": 8,
         "heads": 16, "kv_heads": 4, "dim": 64, "page": 32, "dtype": "f16", "window": 0, "sinks": 0,
         "decay": 0.95},
        # a ready batch's caches cut back to 2,048 tokens
        {"name": "evict_batch", "op": "evict", "seqs": 64, "len": 8192, "ragged": True, "mix": 9, "kv_heads": 8,
         "dim": 128, "page": 64, "dtype": "bf16", "budget": 2048, "sinks": 4, "recent": 256},
        # one very long stream cut back to a twelfth
        {"name": "evict_long", "op": "evict", "seqs": 1, "len": 100_000, "ragged": True, "mix": 10, "kv_heads": 4,
         "dim": 128, "page": 128, "dtype": "bf16", "budget": 8192, "sinks": 16, "recent": 1024},
    ]


HEADS = [(8, 8, 64), (16, 4, 64), (14, 2, 64), (16, 2, 128), (32, 8, 128), (28, 4, 128), (6, 1, 128), (12, 12, 80),
         (10, 10, 96), (5, 5, 40)]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3 * 1024 else n


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        t = top.setdefault(c["op"], [0, 0])
        t[0], t[1] = max(t[0], w["bytes"]), max(t[1], w["flops"])
    op = rng.choice(["rotary", "append", "attend", "attend", "attend", "weigh", "weigh", "evict", "evict"])
    while True:
        c = _draw(rng, op)
        w = work(c)
        if w["bytes"] <= top[op][0] and w["flops"] <= top[op][1]:
            return c


def _draw(rng, op):
    H, K, D = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "f16"])
    if op == "rotary":
        return {"op": op, "tokens": _log(rng, 1, 65_536), "heads": H, "dim": D,
                "dtype": rng.choice(["bf16", "f16", "f32"]), "axes": rng.randint(1, 4),
                "interleaved": rng.random() < 0.5, "inverse": rng.random() < 0.5, "span": _log(rng, 16, 16_384)}
    page = rng.choice([16, 20, 32, 64, 64, 128, 256])
    seqs = _log(rng, 1, 128)
    c = {"op": op, "seqs": seqs, "len": _log(rng, 1, 100_000), "ragged": rng.random() < 0.8,
         "mix": rng.randrange(1 << 30), "kv_heads": K, "dim": D, "page": page, "dtype": dtype}
    while c["len"] * seqs * K * D > 1 << 30:   # at most 4 GB of cache
        c["len"] = (c["len"] + 1) // 2
    if op == "evict":
        budget = max(1, _log(rng, max(1, c["len"] // 16), 2 * c["len"]))
        sinks = min(rng.randint(0, 16), budget)
        return dict(c, budget=budget, sinks=sinks, recent=int(rng.random() * 0.5 * (budget - sinks)))
    new = 1 if rng.random() < 0.4 else _log(rng, 1, 2048)
    while new * seqs > 32_768:
        new = (new + 1) // 2
    c.update(heads=H, new=min(new, c["len"]))
    if op == "append":
        return dict(c, axes=rng.randint(1, 4), span=_log(rng, 16, 16_384))
    c.update(window=0, sinks=0)
    if rng.random() < 0.4:
        c.update(window=_log(rng, 1, c["len"]), sinks=rng.randint(0, 200))
    if op == "weigh":
        c.update(decay=round(rng.uniform(0.8, 1.0), 2))
    return c


def _shape(case):
    """Per sequence: tokens cached after the chunk, and tokens of the chunk."""
    S, top, new = case["seqs"], case["len"], case.get("new", 0)
    rng = np.random.default_rng(case["mix"])
    if not case["ragged"]:
        return [top] * S, [new] * S
    lens = np.exp(rng.uniform(math.log(max(1.0, top / 32)), math.log(top), S)).astype(np.int64)
    lens[0] = top
    news = np.ones(S, np.int64) if new == 1 else rng.integers(0, new + 1, S)
    news[0] = new
    return np.maximum(lens, np.maximum(news, 1)).tolist(), news.tolist()


def _pairs(case):
    """Pairs each axis turns: all of them for one axis, else what is left after equal shares goes to the first."""
    R, n = case["dim"] // 2, case["axes"]
    share = R // n
    return [R - share * (n - 1)] + [share] * (n - 1)


def _seen(L, n, W, sinks):
    """Visible (token, key) pairs of a chunk of n tokens at the end of L cached ones."""
    a = np.arange(L - n, L, dtype=np.int64)
    if W == 0:
        return int((a + 1).sum())
    lo = np.maximum(a - W + 1, 0)
    return int((a - lo + 1 + np.minimum(sinks, lo)).sum())


def _touched(L, n, W, sinks):
    """Cached tokens that some token of the chunk sees."""
    if n == 0:
        return 0
    lo = max(0, L - n - W + 1) if W else 0
    return L - lo + min(sinks, lo)


def work(case):
    op, D = case["op"], case["dim"]
    b = 4 if case["dtype"] == "f32" else 2
    if op == "rotary":
        n = case["tokens"] * case["heads"] * D
        return {"bytes": 2 * n * b + 4 * case["tokens"] * case["axes"], "flops": 3 * n}
    lens, news = _shape(case)
    K = case["kv_heads"]
    if op == "evict":
        kept = sum(min(L, case["budget"]) for L in lens)
        return {"bytes": K * (4 * sum(lens) + kept * (4 * D * b + 8)), "flops": K * sum(lens)}
    T, H = sum(news), case["heads"]
    if op == "append":
        return {"bytes": 2 * T * (H + 2 * K) * D * b + 4 * T * (1 + case["axes"]), "flops": 3 * T * (H + K) * D}
    pairs = sum(_seen(L, n, case["window"], case["sinks"]) for L, n in zip(lens, news))
    keys = sum(_touched(L, n, case["window"], case["sinks"]) for L, n in zip(lens, news))
    if op == "attend":
        return {"bytes": 2 * keys * K * D * b + 2 * T * H * D * b + 4 * T * H, "flops": 4 * D * H * pairs}
    held = sum(lens)
    return {"bytes": keys * K * D * b + T * H * D * b + 4 * T * H + 4 * K * (held + held - T),
            "flops": 2 * D * H * pairs}


# ---------------------------------------------------------------------------- inputs
class State:
    pass


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _i64(x):
    return torch.tensor(np.asarray(x), dtype=torch.int64, device=DEV)


def _positions(case, n, g):
    """Text runs on along every axis; image tokens have a time, a row and a column."""
    pos = torch.randint(0, case["span"], (n, case["axes"]), generator=g, device=DEV, dtype=torch.int32)
    text = torch.rand(n, generator=g, device=DEV) < 0.3
    pos[text] = pos[text][:, :1]
    return pos


@functools.lru_cache(maxsize=None)
def _context(stream):
    import paper_2609_18703_gb300 as ro
    return ro.ro_ctx_create(torch.cuda.current_device(), stream, 1)


def _handle(s, case):
    """What a program that makes the calls keeps: a context, the cache's description, the rotary's."""
    import paper_2609_18703_gb300 as ro
    s.ctx = _context(torch.cuda.current_stream().cuda_stream)
    if "axes" in case:
        s.rope = ro.ro_rope(_pairs(case), base=10_000.0, interleaved=case.get("interleaved", False))
    if "page" in case:
        s.cache = ro.ro_cache(s.k, s.v, s.page_base, s.pages)


def prepare(case, seed):
    s, g = State(), _gen(seed)
    s.case, dt, D = case, DTYPES[case["dtype"]], case["dim"]
    if case["op"] == "rotary":
        s.pos = _positions(case, case["tokens"], g)
        # one tensor's heads among the fused projection's
        fused = torch.randn(case["tokens"], case["heads"] + 2, D, generator=g, device=DEV, dtype=dt)
        s.x = fused[:, : case["heads"]]
        s.out = torch.zeros(case["tokens"], case["heads"], D, device=DEV, dtype=dt)
        if own:
            _handle(s, case)
        return s
    s.lens, s.news = _shape(case)
    S, K, ps = case["seqs"], case["kv_heads"], case["page"]
    held = [-(-L // ps) for L in s.lens]
    kept = [-(-min(L, case["budget"]) // ps) for L in s.lens] if case["op"] == "evict" else [0]
    n_src, n_dst = sum(held), sum(kept)
    pool = n_src + max(1, n_src // 16) + n_dst
    s.first_dst = pool - n_dst
    s.k = torch.randn(pool, K, ps, D, generator=g, device=DEV, dtype=dt)
    s.v = torch.randn(pool, K, ps, D, generator=g, device=DEV, dtype=dt)
    pages = torch.randperm(pool - n_dst, generator=g, device=DEV)[:n_src]
    s.base = np.concatenate([[0], np.cumsum(held)])
    s.page_base, s.pages, s.len = _i64(s.base), pages.to(torch.int32), _i32(s.lens)
    if case["op"] == "evict":
        s.k[s.first_dst:] = 0
        s.v[s.first_dst:] = 0
        s.dst_base = _i64(np.concatenate([[0], np.cumsum(kept)]))
        s.dst_pages = (s.first_dst + torch.randperm(n_dst, generator=g, device=DEV)).to(torch.int32)
        top = max(s.lens)
        s.score = torch.randn(S, K, top, generator=g, device=DEV).mul_(2).exp_()
        s.score[torch.rand(S, K, top, generator=g, device=DEV) < 0.2] = 0   # never looked at
        s.keep = torch.full((S, K, case["budget"]), -1, dtype=torch.int32, device=DEV)
        s.len_out = torch.zeros(S, dtype=torch.int32, device=DEV)
        s.score_out = torch.zeros_like(s.score)
        if own:
            _handle(s, case)
        return s
    H, T = case["heads"], sum(s.news)
    u = torch.randn(K, D, generator=g, device=DEV)
    u = u / u.norm(dim=1, keepdim=True) * (2 * D ** 0.25)
    first = pages[torch.as_tensor(s.base[:-1], device=DEV)]
    s.k[first, :, :4] = u[None, :, None].to(dt)
    # q, k and v lie in one row of the fused projection
    fused = torch.randn(T, H + 2 * K, D, generator=g, device=DEV, dtype=dt)
    s.q, s.k_new, s.v_new = fused[:, :H], fused[:, H:H + K], fused[:, H + K:]
    s.q.add_(u.repeat_interleave(H // K, 0).to(dt))
    s.starts = np.concatenate([[0], np.cumsum(s.news)])
    s.tok_base = _i64(s.starts)
    s.tok_seq = torch.repeat_interleave(torch.arange(S, device=DEV, dtype=torch.int32), _i64(s.news))
    s.max_new = max(s.news)
    if case["op"] == "append":
        s.pos = _positions(case, T, g)
        s.q_out = torch.zeros(T, H, D, device=DEV, dtype=dt)
    else:
        s.scale = 1.0 / math.sqrt(D)
        s.out = torch.zeros(T, H, D, device=DEV, dtype=dt)
        s.lse = torch.zeros(T, H, device=DEV)
        if case["op"] == "weigh":
            s.lse.copy_(_sums(s))
            top = max(s.lens)
            s.past = torch.rand(S, K, top, generator=g, device=DEV)
            s.score = torch.zeros(S, K, top, device=DEV)
    if own:
        _handle(s, case)
    return s


def _sequence(s, i):
    """Sequence i's queries [K, G * n, D], its page indices, and which (row, key) pairs are visible."""
    c, L, n = s.case, s.lens[i], s.news[i]
    K, G, D = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    q = s.q[s.starts[i]: s.starts[i] + n].view(n, K, G, D).permute(1, 2, 0, 3).reshape(K, G * n, D)
    pages = s.pages[s.base[i]: s.base[i + 1]].long()
    a = torch.arange(L - n, L, device=DEV)[:, None]
    j = torch.arange(L, device=DEV)[None]
    seen = j <= a
    if c["window"]:
        seen = seen & ((j > a - c["window"]) | (j < c["sinks"]))
    return q, pages, seen


def _dense(pool, pages, L, h):
    return pool[pages, h].reshape(-1, pool.shape[3])[:L]


def _logits(s, q, pages, seen, h, L):
    x = (q[h].float() @ _dense(s.k, pages, L, h).float().T) * s.scale
    return x.view(-1, *seen.shape).masked_fill(~seen, -math.inf).view(x.shape)


def _sums(s):
    lse = torch.zeros_like(s.lse)
    for i, (L, n) in enumerate(zip(s.lens, s.news)):
        if n == 0:
            continue
        q, pages, seen = _sequence(s, i)
        K = q.shape[0]
        rows = torch.stack([torch.logsumexp(_logits(s, q, pages, seen, h, L), 1) for h in range(K)])
        lse[s.starts[i]: s.starts[i] + n] = rows.view(-1, n).T
    return lse


# ---------------------------------------------------------------------------- the passes
def run(s):
    return (_OWN if own else _PLAIN)[s.case["op"]](s)


def _turn(case, x, pos, inverse=False):
    """x [tokens, heads, dim] in 32 bits, turned by its positions."""
    pairs = _pairs(case)
    R = sum(pairs)
    axis = torch.repeat_interleave(torch.arange(len(pairs), device=DEV), torch.tensor(pairs, device=DEV))
    freq = 10_000.0 ** (-torch.arange(R, device=DEV, dtype=torch.float32) / R)
    theta = pos[:, axis].float() * freq
    if inverse:
        theta = -theta
    cos, sin = theta.cos()[:, None], theta.sin()[:, None]
    if case.get("interleaved"):
        x0, x1 = x[..., 0:2 * R:2], x[..., 1:2 * R:2]
        y = torch.stack([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1).flatten(-2)
    else:
        x0, x1 = x[..., :R], x[..., R:2 * R]
        y = torch.cat([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1)
    return torch.cat([y, x[..., 2 * R:]], -1)


def _plain_rotary(s):
    return _turn(s.case, s.x.float(), s.pos, s.case["inverse"]).to(s.x.dtype)


def _plain_append(s):
    dt, ps = s.k.dtype, s.case["page"]
    seq = s.tok_seq.long()
    n = s.tok_base[1:] - s.tok_base[:-1]
    at = (s.len.long() - n)[seq] + torch.arange(seq.numel(), device=DEV) - s.tok_base[seq]
    page = s.pages.long()[s.page_base[seq] + at // ps]
    s.k[page, :, at % ps] = _turn(s.case, s.k_new.float(), s.pos).to(dt)
    s.v[page, :, at % ps] = s.v_new
    return {"q": _turn(s.case, s.q.float(), s.pos).to(dt), "k": s.k, "v": s.v}


def _plain_attend(s):
    out, lse = torch.zeros_like(s.out), torch.zeros_like(s.lse)
    for i, (L, n) in enumerate(zip(s.lens, s.news)):
        if n == 0:
            continue
        q, pages, seen = _sequence(s, i)
        K, rows, D = q.shape
        o = torch.empty(K, rows, D, device=DEV)
        z = torch.empty(K, rows, device=DEV)
        for h in range(K):
            x = _logits(s, q, pages, seen, h, L)
            m = x.amax(1, keepdim=True)
            x = (x - m).exp_()
            total = x.sum(1, keepdim=True)
            o[h] = (x @ _dense(s.v, pages, L, h).float()) / total
            z[h] = (m + total.log())[:, 0]
        t = slice(s.starts[i], s.starts[i] + n)
        out[t] = o.view(-1, n, D).transpose(0, 1).to(out.dtype)
        lse[t] = z.view(-1, n).T
    return {"out": out, "lse": lse}


def _plain_weigh(s):
    score = torch.zeros_like(s.score)
    for i, (L, n) in enumerate(zip(s.lens, s.news)):
        score[i, :, : L - n] = s.past[i, :, : L - n] * s.case["decay"]
        if n == 0:
            continue
        q, pages, seen = _sequence(s, i)
        z = s.lse[s.starts[i]: s.starts[i] + n].T.reshape(q.shape[0], -1, 1)
        for h in range(q.shape[0]):
            score[i, h, :L] += (_logits(s, q, pages, seen, h, L) - z[h]).exp_().sum(0)
    return score


def _plain_evict(s):
    c, ps = s.case, s.case["page"]
    keep, score = torch.full_like(s.keep, -1), torch.zeros_like(s.score)
    count = [min(L, c["budget"]) for L in s.lens]
    K, at = c["kv_heads"], 0
    heads = torch.arange(K, device=DEV)[:, None]
    for i, (L, n) in enumerate(zip(s.lens, count)):
        if n == L:
            idx = torch.arange(L, device=DEV).expand(K, L)
        else:
            mid = s.score[i, :, c["sinks"]: L - c["recent"]]
            order = torch.sort(mid, dim=1, descending=True, stable=True)[1][:, : n - c["sinks"] - c["recent"]]
            ends = torch.cat([torch.arange(c["sinks"], device=DEV), torch.arange(L - c["recent"], L, device=DEV)])
            idx = torch.cat([ends.expand(K, -1), order + c["sinks"]], 1).sort(1)[0]
        keep[i, :, :n] = idx
        score[i, :, :n] = s.score[i].gather(1, idx)
        src = s.pages[s.base[i]: s.base[i + 1]].long()
        d = torch.arange(n, device=DEV)
        dst = s.dst_pages[at + d // ps].long().expand(K, n)
        for pool in (s.k, s.v):
            pool[dst, heads, (d % ps).expand(K, n)] = pool[src[idx // ps], heads, idx % ps]
        at += -(-n // ps)
    return {"keep": keep, "len": _i32(count), "k": s.k[s.first_dst:], "v": s.v[s.first_dst:], "score": score}


def _call(s, status):
    import paper_2609_18703_gb300 as ro
    if status != ro.RO_OK:
        raise ro.RoError("pass", status, ro.ro_last_error(s.ctx))


def _own_rotary(s):
    import paper_2609_18703_gb300 as ro
    _call(s, ro.ro_rotary(s.ctx, s.x, s.out, s.pos, s.rope, s.case["inverse"]))
    return s.out


def _own_append(s):
    import paper_2609_18703_gb300 as ro
    _call(s, ro.ro_cache_append(s.ctx, s.cache, s.tok_base, s.tok_seq, s.len, s.pos, s.rope, s.q, s.q_out, s.k_new,
                                s.v_new))
    return {"q": s.q_out, "k": s.k, "v": s.v}


def _own_attend(s):
    import paper_2609_18703_gb300 as ro
    c = s.case
    _call(s, ro.ro_cache_attend(s.ctx, s.cache, s.tok_base, s.max_new, s.len, max(s.lens), s.q, s.scale, c["window"],
                                c["sinks"], s.out, s.lse))
    return {"out": s.out, "lse": s.lse}


def _own_weigh(s):
    import paper_2609_18703_gb300 as ro
    c = s.case
    _call(s, ro.ro_cache_weigh(s.ctx, s.cache, s.tok_base, s.max_new, s.len, s.q, s.scale, c["window"], c["sinks"],
                               s.lse, c["decay"], s.past, s.score))
    return s.score


def _own_evict(s):
    import paper_2609_18703_gb300 as ro
    c = s.case
    _call(s, ro.ro_cache_evict(s.ctx, s.cache, s.len, s.score, c["budget"], c["sinks"], c["recent"], s.dst_base,
                               s.dst_pages, s.keep, s.len_out, s.score_out))
    return {"keep": s.keep, "len": s.len_out, "k": s.k[s.first_dst:], "v": s.v[s.first_dst:], "score": s.score_out}


_PLAIN = {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh,
          "evict": _plain_evict}
_OWN = {"rotary": _own_rotary, "append": _own_append, "attend": _own_attend, "weigh": _own_weigh,
        "evict": _own_evict}


# ---------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    if case["op"] in ("attend", "weigh"):   # over the whole of each sequence, unseen keys too
        lens, news = _shape(case)
        if 4 * case["dim"] * case["heads"] * sum(L * n for L, n in zip(lens, news)) > 6e12:
            return None
    global own
    was, own = own, False   # the inputs alone, no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"rotary": _exact_rotary, "append": _exact_append, "attend": _exact_attend, "weigh": _exact_weigh,
            "evict": _exact_evict}[case["op"]](s)


def _exact_turn(case, x, pos, sign):
    y = x.double().clone()
    pairs = _pairs(case)
    R, p = sum(pairs), 0
    for axis, width in enumerate(pairs):
        for _ in range(width):
            theta = sign * pos[:, axis].double() * math.exp(-math.log(10_000.0) * p / R)
            i, j = (2 * p, 2 * p + 1) if case.get("interleaved") else (p, p + R)
            a, b = x[..., i].double(), x[..., j].double()
            c, d = torch.cos(theta)[:, None], torch.sin(theta)[:, None]
            y[..., i] = a * c - b * d
            y[..., j] = b * c + a * d
            p += 1
    return y


def _exact_rotary(s):
    return _exact_turn(s.case, s.x, s.pos, -1.0 if s.case["inverse"] else 1.0)


def _exact_append(s):
    ps = s.case["page"]
    k, v = s.k.double(), s.v.double()
    turned = _exact_turn(s.case, s.k_new, s.pos, 1.0)
    for i, (L, n) in enumerate(zip(s.lens, s.news)):
        for t0 in range(0, n, ps):   # runs of tokens that share at most two pages
            t = np.arange(t0, min(n, t0 + ps))
            at = L - n + t
            page = s.pages[_i64(s.base[i] + at // ps)].long()
            k[page, :, _i64(at % ps)] = turned[_i64(s.starts[i] + t)]
            v[page, :, _i64(at % ps)] = s.v_new[_i64(s.starts[i] + t)].double()
    return {"q": _exact_turn(s.case, s.q, s.pos, 1.0), "k": k, "v": v}


def _exact_rows(s, i, h):
    """The logits in 64 bits of query head h, keys of sequence i, unseen ones at -inf."""
    c, L, n = s.case, s.lens[i], s.news[i]
    kh = h // (c["heads"] // c["kv_heads"])
    slot = torch.arange(L, device=DEV)
    page = s.pages[s.base[i] + slot // c["page"]].long()
    keys, values = s.k[page, kh, slot % c["page"]].double(), s.v[page, kh, slot % c["page"]].double()
    x = torch.einsum("td,jd->tj", s.q[s.starts[i]: s.starts[i] + n, h].double(), keys) / math.sqrt(c["dim"])
    back = torch.arange(L - n, L, device=DEV)[:, None] - slot   # how far behind the token a key lies
    x[back < 0] = -math.inf
    if c["window"]:
        x[(back >= c["window"]) & (slot >= c["sinks"])] = -math.inf
    return x, values


def _exact_attend(s):
    out, lse = s.out.double() * 0, s.lse.double() * 0
    for i, n in enumerate(s.news):
        for h in range(s.case["heads"] if n else 0):
            x, values = _exact_rows(s, i, h)
            t = slice(s.starts[i], s.starts[i] + n)
            lse[t, h] = torch.logsumexp(x, 1)
            out[t, h] = torch.softmax(x, 1) @ values
    return {"out": out, "lse": lse}


def _exact_weigh(s):
    score = s.score.double() * 0
    G = s.case["heads"] // s.case["kv_heads"]
    for i, (L, n) in enumerate(zip(s.lens, s.news)):
        score[i, :, : L - n] = s.past[i, :, : L - n].double() * s.case["decay"]
        for h in range(s.case["heads"] if n else 0):
            x, _ = _exact_rows(s, i, h)
            z = s.lse[s.starts[i]: s.starts[i] + n, h].double()
            score[i, h // G, :L] += torch.exp(x - z[:, None]).sum(0)
    return score


def _exact_evict(s):
    c, ps = s.case, s.case["page"]
    K = c["kv_heads"]
    keep = np.full(tuple(s.keep.shape), -1, np.int64)
    score = torch.zeros(tuple(s.score.shape), dtype=torch.float64, device=DEV)
    weights = s.score.cpu().numpy().astype(np.float64)
    k, v = s.k[s.first_dst:].double(), s.v[s.first_dst:].double()
    count, at = [], 0
    for i, L in enumerate(s.lens):
        n = min(L, c["budget"])
        count.append(n)
        slots = np.arange(n)
        dst = s.dst_pages[_i64(at + slots // ps)].long() - s.first_dst
        for h in range(K):
            if n == L:
                chosen = np.arange(L)
            else:
                lo, hi = c["sinks"], L - c["recent"]
                heavy = np.lexsort((np.arange(lo, hi), -weights[i, h, lo:hi]))[: n - lo - c["recent"]] + lo
                chosen = np.sort(np.concatenate([np.arange(lo), heavy, np.arange(hi, L)]))
            keep[i, h, :n] = chosen
            j = _i64(chosen)
            page = s.pages[s.base[i] + j // ps].long()
            score[i, h, :n] = s.score[i, h, j].double()
            k[dst, h, _i64(slots % ps)] = s.k[page, h, j % ps].double()
            v[dst, h, _i64(slots % ps)] = s.v[page, h, j % ps].double()
        at += -(-n // ps)
    return {"keep": _i32(keep), "len": _i32(count), "k": k, "v": v, "score": score}
