"""The workloads of the operators that a generation step needs beside the paged
cache's own, for timing and for comparing outputs.

  attend   attention over the paged cache whose scores are capped by a tanh, get
           a bias that depends on distance, a document mask or a prefix (frame) mask
  sample   tokens from logits and given random numbers: temperature, top-k,
           top-p and min-p, each row its own
  fork     sequences go on in any number of continuations (none: they end);
           full pages are shared and counted, the open one is copied
  compact  the pages in use move to the low end of the pool

`prepare` makes inputs from the seed alone: normal values, keys and queries with
a common direction on each sequence's first tokens (they draw weight, as first
tokens do), pages in random order, slots past a sequence's length holding another
sequence's old values, logits with a few likely tokens above a wide floor.
Lengths, documents, branches and each row's sampling settings belong to the case
(`mix`), not to the seed.
"""
import functools
import math

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NOTHING = 0x7FFFFFFF   # the first slot of a token that pads a chunk: it sees nothing


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # one user, one token, scores that fall with distance: latency
        {"name": "attend_one", "op": "attend", "seqs": 1, "new": 1, "len": 777, "ragged": False, "mix": 1,
         "heads": 16, "kv_heads": 4, "dim": 64, "page": 16, "dtype": "f16", "window": 0, "sinks": 0,
         "cap": 0.0, "slopes": True, "docs": 0, "frame": 0},
        # single tokens of a ready batch under a cap, caches of 1 to 32 thousand tokens
        {"name": "attend_singles", "op": "attend", "seqs": 64, "new": 1, "len": 32_000, "ragged": True, "mix": 2,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "window": 0, "sinks": 0,
         "cap": 50.0, "slopes": False, "docs": 0, "frame": 0},
        # chunks of long prompts under a cap over what is cached already
        {"name": "attend_chunks", "op": "attend", "seqs": 8, "new": 2048, "len": 16_384, "ragged": True, "mix": 3,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "window": 0, "sinks": 0,
         "cap": 30.0, "slopes": False, "docs": 0, "frame": 0},
        # documents' pages packed into two rows, each page attended by itself, nearer tokens first
        {"name": "attend_documents", "op": "attend", "seqs": 2, "new": 8192, "len": 8192, "ragged": False, "mix": 4,
         "heads": 16, "kv_heads": 2, "dim": 128, "page": 32, "dtype": "f16", "window": 0, "sinks": 0,
         "cap": 0.0, "slopes": True, "docs": 700, "frame": 0},
        # a stream of frames: the tokens of a frame see one another both ways, behind them a window and the first tokens
        {"name": "attend_frames", "op": "attend", "seqs": 4, "new": 729, "len": 20_000, "ragged": True, "mix": 5,
         "heads": 28, "kv_heads": 4, "dim": 128, "page": 128, "dtype": "bf16", "window": 4096, "sinks": 4,
         "cap": 0.0, "slopes": False, "docs": 0, "frame": 243},
        # one user's next token: latency
        {"name": "sample_one", "op": "sample", "rows": 1, "vocab": 32_000, "dtype": "f32", "mix": 11, "pad": 0,
         "temperature": True, "top_k": True, "top_p": True, "min_p": False},
        # a ready batch's next tokens, every request with settings of its own, some greedy
        {"name": "sample_mixed", "op": "sample", "rows": 256, "vocab": 131_072, "dtype": "bf16", "mix": 12, "pad": 0,
         "temperature": True, "top_k": True, "top_p": True, "min_p": True},
        # an odd vocabulary, rows at any alignment, everything above a share of the likeliest
        {"name": "sample_odd", "op": "sample", "rows": 40, "vocab": 100_003, "dtype": "f32", "mix": 13, "pad": 0,
         "temperature": True, "top_k": False, "top_p": False, "min_p": True},
        # a step of a beam search or of parallel samples: branches end, go on and split
        {"name": "fork_beams", "op": "fork", "seqs": 128, "len": 8192, "ragged": True, "mix": 21, "kv_heads": 8,
         "dim": 128, "page": 64, "dtype": "bf16", "layers": 2, "most": 4, "room": 256},
        # one long prompt, 64 samples of it
        {"name": "fork_prompt", "op": "fork", "seqs": 1, "len": 100_003, "ragged": False, "mix": 22, "kv_heads": 4,
         "dim": 64, "page": 16, "dtype": "f16", "layers": 1, "most": 64, "room": 64},
        # a small pool after a few sequences ended: latency
        {"name": "compact_small", "op": "compact", "pages": 300, "used": 0.6, "seqs": 12, "mix": 31, "kv_heads": 2,
         "dim": 64, "page": 32, "dtype": "f16", "layers": 1},
        # a server's pool after many did
        {"name": "compact_pool", "op": "compact", "pages": 20_000, "used": 0.55, "seqs": 300, "mix": 32, "kv_heads": 8,
         "dim": 128, "page": 16, "dtype": "bf16", "layers": 1},
    ]


HEADS = [(8, 8, 64), (16, 4, 64), (14, 2, 64), (16, 2, 128), (32, 8, 128), (28, 4, 128), (6, 1, 128), (12, 12, 80),
         (10, 10, 96), (5, 5, 40)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        t = top.setdefault(c["op"], [0, 0])
        t[0], t[1] = max(t[0], w["bytes"]), max(t[1], w["flops"])
    op = rng.choice(["attend", "attend", "attend", "sample", "sample", "fork", "compact"])
    while True:
        c = _draw(rng, op)
        w = work(c)
        if w["bytes"] <= top[op][0] and w["flops"] <= top[op][1]:
            return c


def _draw(rng, op):
    mix = rng.randrange(1 << 30)
    if op == "sample":
        return {"op": op, "rows": _log(rng, 1, 512), "vocab": _log(rng, 2, 200_000),
                "dtype": rng.choice(["bf16", "f16", "f32"]), "mix": mix, "pad": rng.choice([0, 0, 1, 5, 64]),
                "temperature": rng.random() < 0.8, "top_k": rng.random() < 0.5, "top_p": rng.random() < 0.5,
                "min_p": rng.random() < 0.5}
    H, K, D = rng.choice(HEADS)
    c = {"op": op, "mix": mix, "kv_heads": K, "dim": D, "page": rng.choice([16, 20, 32, 64, 64, 128, 256]),
         "dtype": rng.choice(["bf16", "f16"])}
    if op == "compact":
        c.update(pages=_log(rng, 16, 20_000), used=round(rng.uniform(0.05, 0.98), 2), seqs=_log(rng, 1, 400),
                 layers=rng.randint(1, 3))
        while c["pages"] * c["page"] * c["layers"] * K * D > 1 << 29:
            c["pages"] = (c["pages"] + 1) // 2
        return c
    seqs = _log(rng, 1, 128)
    c.update(seqs=seqs, len=_log(rng, 1, 100_000), ragged=rng.random() < 0.8)
    most = 1 << (28 if op == "fork" else 30)
    while c["len"] * seqs * K * D > most:
        c["len"] = (c["len"] + 1) // 2
    if op == "fork":
        return dict(c, layers=rng.randint(1, 3), most=rng.choice([2, 3, 4, 8, max(1, 256 // seqs)]),
                    room=_log(rng, 1, 300))
    new = 1 if rng.random() < 0.4 else _log(rng, 1, 8192)
    while new * seqs > 32_768:
        new = (new + 1) // 2
    new = min(new, c["len"])
    c.update(heads=H, new=new, window=0, sinks=0, cap=0.0, slopes=rng.random() < 0.4, docs=0, frame=0)
    if rng.random() < 0.5:
        c.update(cap=round(rng.uniform(5.0, 60.0), 1))
    if rng.random() < 0.3:
        c.update(window=_log(rng, 1, c["len"]), sinks=rng.randint(0, 200))
    if rng.random() < 0.3:
        c.update(docs=_log(rng, 1, c["len"]))
    if rng.random() < 0.3:
        c.update(frame=_log(rng, 1, 600))
    if not (c["cap"] or c["slopes"] or c["docs"] or c["frame"]):
        c.update(cap=30.0)
    return c


@functools.lru_cache(maxsize=None)
def _layout(S, top, new, ragged, mix):
    rng = np.random.default_rng(mix)
    if not ragged:
        return [top] * S, [new] * S
    lens = np.exp(rng.uniform(math.log(max(1.0, top / 32)), math.log(top), S)).astype(np.int64)
    lens[0] = top
    news = np.ones(S, np.int64) if new == 1 else rng.integers(0, new + 1, S)
    news[0] = new
    return np.maximum(lens, np.maximum(news, 1)).tolist(), news.tolist()


def _shape(case):
    """Per sequence: tokens cached after the chunk, and tokens of the chunk."""
    return _layout(case["seqs"], case["len"], case.get("new", 0), case["ragged"], case["mix"])


def _masks(case):
    """Per sequence: of each token of the chunk its slot, the first slot it sees and the slot its frame ends before."""
    rng = np.random.default_rng([case["mix"], 1])
    rows = []
    for L, n in zip(*_shape(case)):
        a = np.arange(L - n, L, dtype=np.int64)
        first, until = np.zeros(n, np.int64), np.zeros(n, np.int64)
        if case["docs"]:
            # documents of about `docs` tokens, one after another; a few tokens only pad the chunk
            step = rng.integers(1, 2 * case["docs"] + 1, 2 * (L // case["docs"]) + 8)
            start = np.concatenate([[0], np.cumsum(step)])
            first = start[np.searchsorted(start, a, side="right") - 1]
            first[rng.random(n) < 0.01] = NOTHING
        if case["frame"]:
            until = np.minimum((a // case["frame"] + 1) * case["frame"], L)
        rows.append((a, first, until))
    return rows


def _bounds(case, a, first, until, L):
    """What each token sees: [lo, end) and [first, sink)."""
    end = np.minimum(np.maximum(a + 1, until), L)
    lo = np.maximum(first, a - case["window"] + 1) if case["window"] else first
    sink = np.minimum(first + case["sinks"], lo)
    empty = first > a
    return np.where(empty, 0, lo), np.where(empty, 0, end), np.where(empty, 0, first), np.where(empty, 0, sink)


def _branches(case):
    """Of each sequence how many continuations it has, and the slots each continuation's pages hold beside its tokens."""
    rng = np.random.default_rng([case["mix"], 2])
    S = case["seqs"]
    if S == 1:
        return [case["most"]], [case["room"]] * case["most"]
    kids = rng.choice(case["most"] + 1, S, p=[0.35] + [0.35] + [0.3 / (case["most"] - 1)] * (case["most"] - 1)
                      if case["most"] > 1 else [0.5, 0.5])
    kids[0] = max(1, kids[0])
    return kids.tolist(), rng.integers(0, case["room"] + 1, int(kids.sum())).tolist()


def _settings(case):
    """Each row's temperature, top-k, top-p and min-p."""
    rng = np.random.default_rng([case["mix"], 3])
    n, V = case["rows"], case["vocab"]
    t = np.where(rng.random(n) < (0.1 if n > 1 else 0.0), 0.0, rng.uniform(0.5, 1.3, n)).astype(np.float32)
    k = np.where(rng.random(n) < 0.3, 0, rng.integers(1, min(V, 200) + 1, n)).astype(np.int64)
    p = np.where(rng.random(n) < 0.2, 1.0, rng.uniform(0.5, 0.99, n)).astype(np.float32)
    m = np.where(rng.random(n) < 0.2, 0.0, rng.uniform(0.001, 0.2, n)).astype(np.float32)
    return t, k, p, m


def _pool(case):
    """A pool some of whose pages are in use: each sequence's list (some share their first pages), and the counts."""
    rng = np.random.default_rng([case["mix"], 4])
    n, S = case["pages"], case["seqs"]
    take = max(1, int(round(n * case["used"])))
    free = rng.permutation(n)[:take]
    cuts = np.sort(rng.integers(0, take + 1, S - 1))
    lists = np.split(free, cuts)
    for s in range(1, S):
        if rng.random() < 0.2 and len(lists[s - 1]) > 1:   # a branch: the pages before its own are its neighbour's
            lists[s] = np.concatenate([lists[s - 1][: len(lists[s - 1]) // 2], lists[s]])
    refs = np.zeros(n, np.int64)
    for x in lists:
        np.add.at(refs, x, 1)
    return lists, refs


def _page_bytes(case):
    return 2 * 2 * case["kv_heads"] * case["page"] * case["dim"]   # keys and values


def work(case):
    op, D = case["op"], case.get("dim", 0)
    if op == "sample":
        b = 4 if case["dtype"] == "f32" else 2
        n, V = case["rows"], case["vocab"]
        given = sum(case[x] for x in ("temperature", "top_k", "top_p", "min_p"))
        return {"bytes": n * (V * b + 4 * given + 16), "flops": 4 * n * V}
    if op == "compact":
        lists, refs = _pool(case)
        used = int((refs > 0).sum())
        moved = int((refs[used:] > 0).sum())
        entries = sum(len(x) for x in lists)
        return {"bytes": 2 * moved * case["layers"] * _page_bytes(case) + 8 * case["pages"] + 8 * entries + 8 * moved,
                "flops": case["pages"] + entries}
    lens, news = _shape(case)
    ps = case["page"]
    if op == "fork":
        kids, room = _branches(case)
        old, new, slots, at = sum(-(-L // ps) for L in lens), 0, 0, 0
        for L, n in zip(lens, kids):
            new += sum(-(-(L + r) // ps) for r in room[at: at + n])
            slots += max(0, n - 1) * (L % ps)
            at += n
        pool = _fork_pages(case)
        return {"bytes": 2 * slots * case["layers"] * _page_bytes(case) // ps + 4 * old + 8 * new + 8 * pool
                + 8 * (len(lens) + 3 * sum(kids)), "flops": old + new + pool}
    K, H, T = case["kv_heads"], case["heads"], sum(news)
    pairs = keys = 0
    for L, (a, first, until) in zip(lens, _masks(case)):
        lo, end, f, sink = _bounds(case, a, first, until, L)
        pairs += int((end - lo).sum() + (sink - f).sum())
        seen = np.zeros(L + 1, np.int64)
        for x, y in ((lo, end), (f, sink)):
            np.add.at(seen, x, 1)
            np.add.at(seen, np.maximum(y, x), -1)
        keys += int((np.cumsum(seen) > 0).sum())
    given = T * 4 * ((case["docs"] > 0) + (case["frame"] > 0)) + (4 * H if case["slopes"] else 0)
    return {"bytes": 4 * keys * K * D + 4 * T * H * D + 4 * T * H + given, "flops": 4 * D * H * pairs}


def _fork_pages(case):
    """Pages of a fork's pool: what is held, what the continuations can need, and some."""
    lens, _ = _shape(case)
    kids, room = _branches(case)
    ps = case["page"]
    held, need, at = sum(-(-L // ps) for L in lens), 0, 0
    for L, n in zip(lens, kids):
        need += sum(-(-(L + r) // ps) - L // ps for r in room[at: at + n])
        at += n
    return held + need + max(2, (held + need) // 16)


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


def _offsets(counts):
    return np.concatenate([[0], np.cumsum(np.asarray(counts, np.int64))]).astype(np.int64)


@functools.lru_cache(maxsize=None)
def _context(stream):
    import paper_2609_18703_gb300 as ro
    return ro.ro_ctx_create(torch.cuda.current_device(), stream, 1)


def _handle(s):
    """What a program that makes the calls keeps: a context, the cache's description, the call's settings."""
    import paper_2609_18703_gb300 as ro
    op = s.case["op"]
    s.ctx = _context(torch.cuda.current_stream().cuda_stream)
    if op == "sample":
        s.how = ro.ro_sampling(s.temperature, s.top_k, s.top_p, s.min_p)
    elif op == "attend":
        s.cache = ro.ro_cache(s.k, s.v, s.page_base, s.pages)
        s.bias = ro.ro_bias(s.case["cap"], s.slope, s.first, s.until)
    else:
        s.caches = [ro.ro_cache(k, v, s.page_base, s.pages) for k, v in zip(s.k, s.v)]
        s.moves = ro.ro_moves(s.move_from, s.move_to, s.move_slots, s.n_moves)


def prepare(case, seed):
    s, g = State(), _gen(seed)
    s.case = case
    {"attend": _prepare_attend, "sample": _prepare_sample, "fork": _prepare_fork, "compact": _prepare_compact}[
        case["op"]](s, case, g)
    if own:
        _handle(s)
    return s


def _prepare_attend(s, case, g):
    dt, D, ps = DTYPES[case["dtype"]], case["dim"], case["page"]
    S, K, H = case["seqs"], case["kv_heads"], case["heads"]
    s.lens, s.news = _shape(case)
    held = [-(-L // ps) for L in s.lens]
    n = sum(held)
    pool = n + max(1, n // 16)
    s.k = torch.randn(pool, K, ps, D, generator=g, device=DEV, dtype=dt)
    s.v = torch.randn(pool, K, ps, D, generator=g, device=DEV, dtype=dt)
    pages = torch.randperm(pool, generator=g, device=DEV)[:n]
    s.base = _offsets(held)
    s.page_base, s.pages, s.len = _i64(s.base), pages.to(torch.int32), _i32(s.lens)
    T = sum(s.news)
    u = torch.randn(K, D, generator=g, device=DEV)
    u = u / u.norm(dim=1, keepdim=True) * (2 * D ** 0.25)
    at = torch.as_tensor(s.base[:-1], device=DEV)
    s.k[pages[at], :, :4] = u[None, :, None].to(dt)
    # the queries lie in the rows of the fused projection
    fused = torch.randn(T, H + 2 * K, D, generator=g, device=DEV, dtype=dt)
    s.q = fused[:, :H]
    s.q.add_(u.repeat_interleave(H // K, 0).to(dt))
    s.starts = _offsets(s.news)
    s.tok_base, s.max_new, s.scale = _i64(s.starts), max(s.news), 1.0 / math.sqrt(D)
    masks = _masks(case)
    s.first = _i32(np.concatenate([m[1] for m in masks])) if case["docs"] else None
    s.until = _i32(np.concatenate([m[2] for m in masks])) if case["frame"] else None
    # a head's slope halves from head to head, over eight halvings
    s.slope = (2.0 ** (-8.0 * torch.arange(1, H + 1, device=DEV) / H)).float() if case["slopes"] else None
    s.out = torch.zeros(T, H, D, device=DEV, dtype=dt)
    s.lse = torch.zeros(T, H, device=DEV)


def _prepare_sample(s, case, g):
    n, V = case["rows"], case["vocab"]
    x = torch.randn(n, V + case["pad"], generator=g, device=DEV).mul_(1.5)
    # a few likely tokens, each row its own
    likely = torch.randint(0, V, (n, 24), generator=g, device=DEV)
    x.scatter_add_(1, likely, 4.0 + 2.5 * torch.randn(n, 24, generator=g, device=DEV))
    if V > 64:   # tokens that the grammar rules out
        x[:, 5:5 + V // 50] = -math.inf
    s.logits = x.to(DTYPES[case["dtype"]])[:, :V]
    t, k, p, m = _settings(case)
    s.temperature = torch.tensor(t, device=DEV) if case["temperature"] else None
    s.top_k = _i32(k) if case["top_k"] else None
    s.top_p = torch.tensor(p, device=DEV) if case["top_p"] else None
    s.min_p = torch.tensor(m, device=DEV) if case["min_p"] else None
    s.u = torch.rand(n, generator=g, device=DEV)
    s.token, s.kept = (torch.zeros(n, dtype=torch.int32, device=DEV) for _ in range(2))
    s.logp = torch.zeros(n, device=DEV)


def _pools(s, case, g, n):
    dt = DTYPES[case["dtype"]]
    size = (n, case["kv_heads"], case["page"], case["dim"])
    s.k = [torch.randn(size, generator=g, device=DEV, dtype=dt) for _ in range(case["layers"])]
    s.v = [torch.randn(size, generator=g, device=DEV, dtype=dt) for _ in range(case["layers"])]


def _moves(s, n):
    s.move_from, s.move_to, s.move_slots = (torch.full((max(n, 1),), -1, dtype=torch.int32, device=DEV) for _ in range(3))
    s.n_moves = torch.zeros(1, dtype=torch.int32, device=DEV)


def _prepare_fork(s, case, g):
    ps = case["page"]
    s.lens, _ = _shape(case)
    s.kids, room = _branches(case)
    n = _fork_pages(case)
    held = [-(-L // ps) for L in s.lens]
    order = torch.randperm(n, generator=g, device=DEV)[: sum(held)].to(torch.int32)
    s.base = _offsets(held)
    lists = [order[s.base[i]: s.base[i + 1]] for i in range(len(held))]
    for i in range(1, len(held), 3):   # branches of an earlier step: their first pages are their neighbour's
        both = min(s.lens[i], s.lens[i - 1]) // ps // 2
        lists[i] = torch.cat([lists[i - 1][:both], lists[i][both:]])
    s.pages = torch.cat(lists)
    s.page_base, s.len = _i64(s.base), _i32(s.lens)
    s.refs = torch.zeros(n, dtype=torch.int32, device=DEV)
    s.refs.index_add_(0, s.pages.long(), torch.ones_like(s.pages))
    _pools(s, case, g, n)
    s.child_base = _i64(_offsets(s.kids))
    s.child_parent = torch.repeat_interleave(torch.arange(len(s.kids), device=DEV, dtype=torch.int32), _i64(s.kids))
    lens = np.repeat(s.lens, s.kids)
    s.want = (-(-(lens + np.asarray(room, np.int64)) // ps)).tolist()   # pages of each continuation
    s.dst_base = _i64(_offsets(s.want))
    s.dst_seq = torch.repeat_interleave(torch.arange(len(s.want), device=DEV, dtype=torch.int32), _i64(s.want))
    s.dst_pages = torch.full((max(1, sum(s.want)),), -1, dtype=torch.int32, device=DEV)
    s.len_out = torch.zeros(len(s.want), dtype=torch.int32, device=DEV)
    s.refs_out = torch.zeros_like(s.refs)
    _moves(s, len(s.want))


def _prepare_compact(s, case, g):
    lists, refs = _pool(case)
    _pools(s, case, g, case["pages"])
    s.base = _offsets([len(x) for x in lists])
    s.page_base, s.pages = _i64(s.base), _i32(np.concatenate(lists))
    s.refs = _i32(refs)
    s.refs_out, s.pages_out = torch.zeros_like(s.refs), torch.zeros_like(s.pages)
    s.n_used = torch.zeros(1, dtype=torch.int32, device=DEV)
    _moves(s, (case["pages"] + 1) // 2)


# ---------------------------------------------------------------------------- the passes
def run(s):
    return (_OWN if own else _PLAIN)[s.case["op"]](s)


def _plain_attend(s):
    c = s.case
    K, G, D = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    out, lse = torch.zeros_like(s.out), torch.full_like(s.lse, -math.inf)
    for i, (L, n) in enumerate(zip(s.lens, s.news)):
        if n == 0:
            continue
        t = slice(s.starts[i], s.starts[i] + n)
        pages = s.pages[s.base[i]: s.base[i + 1]].long()
        a = torch.arange(L - n, L, device=DEV)[:, None]
        j = torch.arange(L, device=DEV)[None]
        first = s.first[t].long()[:, None] if s.first is not None else torch.zeros_like(a)
        until = s.until[t].long()[:, None] if s.until is not None else torch.zeros_like(a)
        seen = (j >= first) & (j < torch.maximum(a + 1, until)) & (first <= a)
        if c["window"]:
            seen &= (j > a - c["window"]) | (j < first + c["sinks"])
        some = seen.any(1).repeat(G)[:, None]
        apart = (a - j).abs().float()
        q = s.q[t].view(n, K, G, D).permute(1, 2, 0, 3).reshape(K, G * n, D)
        o, z = torch.empty(K, G * n, D, device=DEV), torch.empty(K, G * n, device=DEV)
        for h in range(K):
            keys, values = (pool[pages, h].reshape(-1, D)[:L].float() for pool in (s.k, s.v))
            x = (q[h].float() @ keys.T) * s.scale
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            x = x.view(G, n, L)
            if s.slope is not None:
                x = x - s.slope[h * G: (h + 1) * G, None, None] * apart
            x = x.masked_fill(~seen, -math.inf).view(G * n, L)
            m = x.amax(1, keepdim=True).masked_fill(~some, 0.0)
            x = (x - m).exp_()
            total = x.sum(1, keepdim=True)
            o[h] = ((x @ values) / total).masked_fill(~some, 0.0)
            z[h] = (m + total.log())[:, 0]
        out[t] = o.view(-1, n, D).transpose(0, 1).to(out.dtype)
        lse[t] = z.view(-1, n).T
    return {"out": out, "lse": lse}


def _plain_sample(s):
    """In 64 bits: a sum next to a border decides which token it is."""
    x = s.logits.double()
    n, V = x.shape
    one = torch.ones(n, 1, dtype=torch.float64, device=DEV)
    t = s.temperature.double()[:, None] if s.temperature is not None else one
    top_p = s.top_p.double()[:, None] if s.top_p is not None else one
    min_p = s.min_p.double()[:, None] if s.min_p is not None else one * 0
    order = torch.sort(x, dim=1, descending=True, stable=True)
    value, index = order.values, order.indices
    rank = torch.arange(V, device=DEV)[None]
    greedy = t == 0
    w = torch.exp((value - value[:, :1]) / torch.where(greedy, one, t))
    keep = (value > -math.inf) & (~greedy | (rank == 0))
    if s.top_k is not None:
        k = s.top_k.long()[:, None]
        keep &= (k == 0) | (rank < k)
    mass = w * keep
    ahead = mass.cumsum(1) - mass
    keep &= (top_p >= 1) | (ahead < top_p * mass.sum(1, keepdim=True)) | (rank == 0)
    keep &= w >= min_p
    kept = torch.zeros_like(keep).scatter_(1, index, keep)
    w = torch.zeros_like(w).scatter_(1, index, w * keep)
    run = w.cumsum(1)
    total = run[:, -1:]
    token = (kept & (run > s.u.double()[:, None] * total)).int().argmax(1)
    logp = (w.gather(1, token[:, None]) / total).log()[:, 0]
    return {"token": token.int(), "logp": logp.float(), "kept": kept.sum(1).int()}


def _fill(x, values):
    x[: values.numel()] = values.to(x.dtype)


def _plain_fork(s):
    ps = s.case["page"]
    full = (s.len // ps).long()
    free = torch.nonzero(s.refs == 0)[:, 0]
    child = s.dst_seq.long()
    parent = s.child_parent.long()[child]
    at = torch.arange(child.numel(), device=DEV) - s.dst_base[child]   # the page's place in its list
    held = s.page_base[parent + 1] - s.page_base[parent]
    oldest = child == s.child_base[parent]                             # the first continuation keeps the open pages
    there = at < held
    old = s.pages.long()[torch.where(there, s.page_base[parent] + at, 0)]
    keep = there & ((at < full[parent]) | (oldest & (s.refs[old] == 1)))
    fresh = ~keep
    page = torch.where(keep, old, free[torch.where(fresh, fresh.cumsum(0) - 1, 0)])
    s.dst_pages[:] = page.to(torch.int32)
    s.refs_out.copy_(s.refs)
    s.refs_out.index_add_(0, page, torch.ones_like(s.dst_pages))
    s.refs_out.index_add_(0, s.pages.long(), -torch.ones_like(s.pages))
    s.len_out.copy_(s.len[s.child_parent.long()])
    rest = (s.len % ps).long()[parent]
    move = torch.nonzero(fresh & there & (at == full[parent]) & (rest > 0))[:, 0]
    _fill(s.move_from, old[move])
    _fill(s.move_to, page[move])
    _fill(s.move_slots, rest[move])
    s.n_moves.fill_(move.numel())
    slot = torch.arange(ps, device=DEV)
    which, slot = torch.nonzero(slot[None] < rest[move][:, None], as_tuple=True)
    for pool in s.k + s.v:
        pool[page[move][which], :, slot] = pool[old[move][which], :, slot]
    return _forked(s)


def _forked(s):
    return {"pages": s.dst_pages, "refs": s.refs_out, "len": s.len_out, "from": s.move_from, "to": s.move_to,
            "slots": s.move_slots, "moves": s.n_moves, "k": s.k, "v": s.v}


def _plain_compact(s):
    used = s.refs > 0
    index = torch.arange(s.refs.numel(), device=DEV)
    U = used.sum()
    src = torch.nonzero(used & (index >= U))[:, 0]
    dst = torch.nonzero(~used & (index < U))[:, 0]
    place = index.clone()
    place[src] = dst
    s.pages_out.copy_(place[s.pages.long()])
    s.refs_out.copy_(torch.where(index < U, s.refs, 0))
    s.refs_out[dst] = s.refs[src]
    s.n_used.copy_(U)
    _fill(s.move_from, src)
    _fill(s.move_to, dst)
    _fill(s.move_slots, torch.full_like(src, s.case["page"]))
    s.n_moves.fill_(src.numel())
    for pool in s.k + s.v:
        pool[dst] = pool[src]
    return _compacted(s)


def _compacted(s):
    return {"pages": s.pages_out, "refs": s.refs_out, "used": s.n_used, "from": s.move_from, "to": s.move_to,
            "slots": s.move_slots, "moves": s.n_moves, "k": s.k, "v": s.v}


def _call(s, status):
    import paper_2609_18703_gb300 as ro
    if status != ro.RO_OK:
        raise ro.RoError("pass", status, ro.ro_last_error(s.ctx))


def _own_attend(s):
    import paper_2609_18703_gb300 as ro
    c = s.case
    _call(s, ro.ro_cache_attend_biased(s.ctx, s.cache, s.tok_base, s.max_new, s.len, max(s.lens), s.q, s.scale,
                                       c["window"], c["sinks"], s.bias, s.out, s.lse))
    return {"out": s.out, "lse": s.lse}


def _own_sample(s):
    import paper_2609_18703_gb300 as ro
    _call(s, ro.ro_sample(s.ctx, s.logits, s.how, s.u, s.token, s.logp, s.kept))
    return {"token": s.token, "logp": s.logp, "kept": s.kept}


def _own_fork(s):
    import paper_2609_18703_gb300 as ro
    _call(s, ro.ro_cache_fork(s.ctx, s.caches[0], s.len, s.child_base, s.child_parent, s.dst_base, s.dst_seq,
                              s.dst_pages, s.len_out, s.refs, s.refs_out, s.moves))
    for cache in s.caches[1:]:
        _call(s, ro.ro_cache_copy(s.ctx, cache, s.moves))
    return _forked(s)


def _own_compact(s):
    import paper_2609_18703_gb300 as ro
    _call(s, ro.ro_cache_compact(s.ctx, s.caches[0], s.pages_out, s.refs, s.refs_out, s.n_used, s.moves))
    for cache in s.caches[1:]:
        _call(s, ro.ro_cache_copy(s.ctx, cache, s.moves))
    return _compacted(s)


_PLAIN = {"attend": _plain_attend, "sample": _plain_sample, "fork": _plain_fork, "compact": _plain_compact}
_OWN = {"attend": _own_attend, "sample": _own_sample, "fork": _own_fork, "compact": _own_compact}


# ---------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    if case["op"] == "attend":   # over the whole of each sequence, unseen keys too
        lens, news = _shape(case)
        if 4 * case["dim"] * case["heads"] * sum(L * n for L, n in zip(lens, news)) > 6e12:
            return None
    global own
    was, own = own, False   # the inputs alone, no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"attend": _exact_attend, "sample": _exact_sample, "fork": _exact_fork, "compact": _exact_compact}[
        case["op"]](s)


def _exact_attend(s):
    c, masks = s.case, _masks(s.case)
    out, lse = s.out.double() * 0, s.lse.double() - math.inf
    for i, (L, n) in enumerate(zip(s.lens, s.news)):
        if n == 0:
            continue
        slot = np.arange(L)
        a, first, until = masks[i]
        back = a[:, None] - slot
        hidden = (back < 0) & (slot >= until[:, None])
        if c["window"]:
            hidden |= (back >= c["window"]) & (slot - first[:, None] >= c["sinks"])
        hidden |= slot < first[:, None]
        hidden[first > a] = True
        hidden, back = torch.tensor(hidden, device=DEV), torch.tensor(np.abs(back), device=DEV).double()
        place = _i64(slot)
        page = s.pages[s.base[i] + place // c["page"]].long()
        t = slice(s.starts[i], s.starts[i] + n)
        for h in range(c["heads"]):
            kh = h // (c["heads"] // c["kv_heads"])
            keys, values = (p[page, kh, place % c["page"]].double() for p in (s.k, s.v))
            x = torch.einsum("td,jd->tj", s.q[t, h].double(), keys) / math.sqrt(c["dim"])
            if c["cap"] > 0:
                x = torch.tanh(x.div_(c["cap"])) * c["cap"]
            if c["slopes"]:
                x = x - float(s.slope[h]) * back
            x[hidden] = -math.inf
            lse[t, h] = torch.logsumexp(x, 1)
            out[t, h] = torch.nan_to_num(torch.softmax(x, 1), nan=0.0) @ values
    return {"out": out, "lse": lse}


def _exact_sample(s):
    """Row by row on the host, from the likeliest token down."""
    logits = s.logits.float().cpu().numpy().astype(np.float64)
    n, V = logits.shape
    give = lambda x, d: np.full(n, d) if x is None else x.cpu().numpy().astype(np.float64)   # noqa: E731
    t, k, p, m = give(s.temperature, 1.0), give(s.top_k, 0), give(s.top_p, 1.0), give(s.min_p, 0.0)
    u = s.u.cpu().numpy().astype(np.float64)
    token, kept, logp = np.zeros(n, np.int64), np.zeros(n, np.int64), np.zeros(n)
    for r in range(n):
        order = np.lexsort((np.arange(V), -logits[r]))
        order = order[: int(np.isfinite(logits[r]).sum())]
        if t[r] == 0:
            order = order[:1]
        elif 0 < k[r] < order.size:
            order = order[: int(k[r])]
        w = np.exp((logits[r, order] - logits[r, order[0]]) / (t[r] if t[r] else 1.0))
        count = order.size
        if p[r] < 1:
            below = np.concatenate([[0.0], np.cumsum(w)[:-1]]) < p[r] * math.fsum(w)
            count = max(1, int(below.sum()))
        count = min(count, int((w >= m[r]).sum()))
        order, w = order[:count], w[:count]
        place = np.argsort(order)
        runs = np.cumsum(w[place])
        hit = place[int(np.searchsorted(runs, u[r] * runs[-1], side="right"))]
        token[r], kept[r], logp[r] = order[hit], count, math.log(w[hit] / runs[-1])
    return {"token": _i32(token), "logp": torch.tensor(logp, device=DEV), "kept": _i32(kept)}


def _exact_fork(s):
    ps = s.case["page"]
    refs, pages = s.refs.cpu().numpy().astype(np.int64), s.pages.cpu().numpy()
    free = iter(np.flatnonzero(refs == 0).tolist())
    after, lists, moves, lens = refs.copy(), [], [], []
    np.subtract.at(after, pages, 1)
    child = 0
    for i, kids in enumerate(s.kids):
        mine = pages[s.base[i]: s.base[i + 1]].tolist()
        full, rest = divmod(s.lens[i], ps)
        for k in range(kids):
            new = []
            for e in range(s.want[child]):
                if e < full or (k == 0 and e < len(mine) and refs[mine[e]] == 1):
                    new.append(mine[e])
                else:
                    new.append(next(free))
                    if e == full and rest:
                        moves.append((mine[e], new[e], rest))
            np.add.at(after, new, 1)
            lists += new
            lens.append(s.lens[i])
            child += 1
    for x, y, rest in moves:
        for pool in s.k + s.v:
            pool[y, :, :rest] = pool[x, :, :rest]
    return {"pages": _i32(lists if lists else [-1]), "refs": _i32(after), "len": _i32(lens), **_moved(s, moves)}


def _moved(s, moves):
    cols = np.full((3, s.move_from.numel()), -1, np.int64)
    if moves:
        cols[:, : len(moves)] = np.array(moves, np.int64).T
    return {"from": _i32(cols[0]), "to": _i32(cols[1]), "slots": _i32(cols[2]), "moves": _i32([len(moves)]),
            "k": [p.double() for p in s.k], "v": [p.double() for p in s.v]}


def _exact_compact(s):
    refs, pages = s.refs.cpu().numpy(), s.pages.cpu().numpy()
    used = int((refs > 0).sum())
    holes = [i for i in range(used) if refs[i] == 0]
    late = [i for i in range(used, refs.size) if refs[i] > 0]
    place = dict(zip(late, holes))
    after = np.zeros_like(refs)
    for i in np.flatnonzero(refs):
        after[place.get(int(i), int(i))] = refs[i]
    for x, y in place.items():
        for pool in s.k + s.v:
            pool[y] = pool[x]
    return {"pages": _i32([place.get(int(x), int(x)) for x in pages]), "refs": _i32(after), "used": _i32([used]),
            **_moved(s, [(x, y, s.case["page"]) for x, y in place.items()])}
