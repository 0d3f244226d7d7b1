"""Forking, releasing, compacting and copying pages of a cache on the GPU
against the definitions, entry by entry: every output is a whole number or a
copied byte, so everything is equal."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


import paper_2609_18703_gb300 as ro  # noqa: E402

NONE = -1   # RO_NO_PAGE as a signed integer


@pytest.fixture
def ctx():
    c = ro.ro_ctx_create(0, torch.cuda.current_stream(), 1)
    yield c
    ro.ro_ctx_destroy(c)


def ok(ctx, status):
    assert status == ro.RO_OK, ro.ro_last_error(ctx)


def i64(x):
    return torch.as_tensor(np.asarray(x, np.int64)).cuda()


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int64)).to(torch.int32).cuda()


def offsets(counts):
    return np.concatenate([[0], np.cumsum(np.asarray(counts, np.int64))]).astype(np.int64)


def fork(lists, lens, kids, rooms, refs, page):
    """The definition: new lists, lengths, counts, copies, and whether pages ran out."""
    free = iter([p for p in range(len(refs)) if refs[p] == 0])
    after = refs.copy()
    for mine in lists:
        for p in mine:
            after[p] -= 1
    new, lens_out, moves, short, child = [], [], [], False, 0
    for mine, n, k in zip(lists, lens, kids):
        full, rest = divmod(n, page)
        for c in range(k):
            entries = []
            for e in range(rooms[child]):
                if e < full or (c == 0 and e < len(mine) and refs[mine[e]] == 1):
                    entries.append(mine[e])
                    continue
                p = next(free, NONE)
                short |= p == NONE
                entries.append(p)
                if e == full and rest and p != NONE:
                    moves.append((mine[e], p, rest))
            for p in entries:
                if p != NONE:
                    after[p] += 1
            new.append(entries)
            lens_out.append(min(n, rooms[child] * page))
            child += 1
    return new, lens_out, after, moves, short


class Pool:
    def __init__(self, n, heads, page, dim, layers=1, seed=0, dtype=torch.bfloat16, fused=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = [], []
        for _ in range(layers):
            if fused:   # slots of all heads side by side
                both = torch.randn(2, n, page, heads, dim, generator=g, device="cuda").to(dtype)
                k, v = both[0].transpose(1, 2), both[1].transpose(1, 2)
            else:
                k, v = (torch.randn(n, heads, page, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
            self.k.append(k)
            self.v.append(v)
        self.before = [x.clone() for x in self.k + self.v]

    def caches(self, base, pages):
        return [ro.ro_cache(k, v, base, pages) for k, v in zip(self.k, self.v)]

    def check(self, moves):
        for got, old in zip(self.k + self.v, self.before):
            want = old.clone()
            for a, b, n in moves:
                want[b, :, :n] = old[a, :, :n]
            assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def moves_of(cap):
    t = [torch.full((max(cap, 1),), -7, dtype=torch.int32, device="cuda") for _ in range(3)]
    return t, torch.full((1,), -7, dtype=torch.int32, device="cuda")


def run_fork(ctx, lists, lens, kids, rooms, refs, pool, page, in_place=False, expect=None, stream_sync=True):
    base, pages = i64(offsets([len(x) for x in lists])), i32([p for x in lists for p in x] or [0])
    caches = pool.caches(base, pages)
    n = int(sum(kids))
    dst_pages = torch.full((max(1, sum(rooms)),), -7, dtype=torch.int32, device="cuda")[:sum(rooms)]
    len_out = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    refs_d = i32(refs)
    refs_out = refs_d if in_place else torch.full_like(refs_d, -7)
    t, n_moves = moves_of(n)
    moves = ro.ro_moves(*t, n_moves)
    parent = i32(np.repeat(np.arange(len(lists)), kids))
    seq = i32(np.repeat(np.arange(n), rooms))
    ok(ctx, ro.ro_cache_fork(ctx, caches[0], i32(lens), i64(offsets(kids)), parent, i64(offsets(rooms)), seq, dst_pages,
                             len_out, refs_d, refs_out, moves))
    for c in caches[1:]:
        ok(ctx, ro.ro_cache_copy(ctx, c, moves))
    st = ro.ro_ctx_sync(ctx)
    new, want_len, after, want_moves, short = fork(lists, lens, kids, rooms, refs, page)
    tight = any(a < b for a, b in zip(want_len, np.repeat(lens, kids)))
    assert st == (ro.RO_E_CAPACITY if short or tight else ro.RO_OK)
    assert dst_pages.tolist() == [p for x in new for p in x]
    assert len_out.tolist() == want_len
    assert refs_out.tolist() == after.tolist()
    assert n_moves.item() == len(want_moves)
    got = list(zip(*[x[:len(want_moves)].tolist() for x in t]))
    assert got == [tuple(m) for m in want_moves]
    for x in t:
        assert bool((x[len(want_moves):] == -7).all())
    pool.check(want_moves)
    return new


def some_lists(g, n_pages, lens, page, extra=2, share=0.4):
    """Page lists for the lengths, some sharing their first full pages with an earlier one, and the counts."""
    order = iter(g.permutation(n_pages).tolist())
    lists, refs = [], np.zeros(n_pages, np.int64)
    for s, n in enumerate(lens):
        held = -(-n // page) + int(g.integers(0, extra + 1))
        mine = []
        if s and g.random() < share:
            o = int(g.integers(0, s))
            both = min(n, lens[o]) // page
            mine = lists[o][:int(g.integers(0, both + 1))]
        mine = mine + [next(order) for _ in range(held - len(mine))]
        lists.append(mine)
        for p in mine:
            refs[p] += 1
    return lists, refs


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seqs,top,page,heads,dim,layers,fused", [(1, 1, 16, 1, 8, 1, False), (5, 100, 16, 2, 64, 2, False),
                                                                  (40, 300, 7, 3, 40, 1, True), (300, 60, 1, 1, 8, 1, False),
                                                                  (17, 900, 64, 2, 128, 3, True), (3, 5000, 4, 1, 16, 1, False)])
def test_fork(ctx, seqs, top, page, heads, dim, layers, fused, in_place):
    g = np.random.default_rng(seqs + top)
    lens = [int(x) for x in g.integers(0, top + 1, seqs)]
    lens[0] = top
    lists, refs = some_lists(g, 4 * sum(-(-n // page) + 3 for n in lens) + 40, lens, page)
    kids = g.choice([0, 1, 2, 3], seqs).tolist()
    kids[0] = max(kids[0], 1)
    rooms = [-(-lens[s] // page) + int(g.integers(0, 4)) for s in range(seqs) for _ in range(kids[s])]
    # what else holds pages: another cache's lists
    refs[g.integers(0, len(refs), 5)] += 1
    pool = Pool(len(refs), heads, page, dim, layers, fused=fused)
    run_fork(ctx, lists, lens, kids, rooms, refs, pool, page, in_place)


def test_fork_of_an_empty_root_and_ends(ctx):
    """New sequences are the continuations of one that holds nothing; sequences without continuations are released."""
    refs = np.zeros(30, np.int64)
    refs[[3, 7, 8, 9]] = 1
    lists, lens = [[], [3, 7], [8, 9]], [0, 30, 20]
    pool = Pool(30, 2, 16, 64)
    run_fork(ctx, lists, lens, [4, 0, 1], [2, 0, 3, 1, 2], refs, pool, 16)
    run_fork(ctx, lists, lens, [0, 0, 0], [], refs, Pool(30, 2, 16, 64), 16)


def test_fork_whose_open_page_is_shared(ctx):
    """A sequence cut back into a page that another one also holds writes there no longer: every continuation copies."""
    refs = np.zeros(20, np.int64)
    lists, lens = [[4, 5, 6], [4, 5, 9]], [20, 48]   # the first one cut back into page 5
    for x in lists:
        for p in x:
            refs[p] += 1
    new = run_fork(ctx, lists, lens, [2, 1], [3, 3, 3], refs, Pool(20, 1, 16, 32), 16)
    assert new[0][:2] == [4, 0] and new[0][2] == 6 and new[1][:1] == [4] and new[2] == [4, 5, 9]


def test_fork_without_enough_pages_or_room_is_recorded(ctx):
    refs = np.zeros(9, np.int64)
    lists, lens = [[1, 3], [5]], [30, 10]
    for x in lists:
        for p in x:
            refs[p] += 1
    run_fork(ctx, lists, lens, [2, 3], [3, 3, 2, 2, 2], refs, Pool(9, 1, 16, 32), 16)   # 10 wanted, 6 free
    run_fork(ctx, lists, lens, [2, 1], [3, 1, 1], refs, Pool(9, 1, 16, 32), 16)         # a room of 16 for 30 tokens
    run_fork(ctx, lists, lens, [2, 1], [3, 3, 1], refs, Pool(9, 1, 16, 32), 16)


def test_fork_records_what_is_out_of_bounds(ctx):
    pool = Pool(12, 1, 16, 32)
    pages = i32([1, 3, 5])
    base, refs = i64([0, 2, 3]), i32([0, 1, 0, 1, 0, 1] + [0] * 6)

    def call(pages=pages, base=base, refs=refs, parent=(0, 0, 1), child_base=(0, 2, 3), dst_base=(0, 3, 6, 7),
             seq=(0, 0, 0, 1, 1, 1, 2), lens=(20, 10)):
        t, n = moves_of(3)
        out = torch.full((7,), -7, dtype=torch.int32, device="cuda")
        after = torch.zeros_like(refs)
        ok(ctx, ro.ro_cache_fork(ctx, pool.caches(base, pages)[0], i32(lens), i64(child_base), i32(parent), i64(dst_base),
                                 i32(seq), out, torch.zeros(3, dtype=torch.int32, device="cuda"), refs, after, ro.ro_moves(*t, n)))
        return ro.ro_ctx_sync(ctx), out.tolist(), after.tolist()

    st, good, _ = call()
    assert st == ro.RO_OK and good == [1, 3, 0, 1, 2, 4, 5]
    assert call(pages=i32([1, 99, 5]))[0] == ro.RO_E_INVAL
    st, out, _ = call(parent=(0, 9, 1))
    assert st == ro.RO_E_INVAL and out[3:6] == [NONE] * 3
    assert call(seq=(0, 0, 0, 1, 8, 1, 2))[0] == ro.RO_E_INVAL
    assert call(dst_base=(0, 3, 60, 7))[0] == ro.RO_E_INVAL
    assert call(base=i64([0, 90, 3]))[0] == ro.RO_E_INVAL
    assert call(lens=(-5, 10))[0] == ro.RO_E_INVAL
    assert call(lens=(200, 10))[0] == ro.RO_E_CAPACITY
    st, _, after = call(refs=i32([0, 1, 0, 0, 0, 1] + [0] * 6))   # page 3 counted too low
    assert st == ro.RO_E_INVAL
    assert call()[:2] == (ro.RO_OK, good)


def compact(lists, refs):
    used = int((refs > 0).sum())
    late = [p for p in range(used, len(refs)) if refs[p] > 0]
    holes = [p for p in range(used) if refs[p] == 0]
    place = dict(zip(late, holes))
    after = refs.copy()
    for a, b in place.items():
        after[b], after[a] = refs[a], 0
    return [place.get(p, p) for x in lists for p in x], after, used, list(zip(late, holes))


def run_compact(ctx, lists, refs, pool, page, in_place=False):
    base, pages = i64(offsets([len(x) for x in lists])), i32([p for x in lists for p in x] or [0])
    caches = pool.caches(base, pages)
    t, n_moves = moves_of(len(refs) // 2)
    if len(refs) // 2 == 0:
        t = [x[:0] for x in t]
    moves = ro.ro_moves(*t, n_moves)
    refs_d = i32(refs)
    refs_out = refs_d if in_place else torch.full_like(refs_d, -7)
    pages_out = pages if in_place else torch.full_like(pages, -7)
    used = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    ok(ctx, ro.ro_cache_compact(ctx, caches[0], pages_out, refs_d, refs_out, used, moves))
    for c in caches[1:]:
        ok(ctx, ro.ro_cache_copy(ctx, c, moves))
    ok(ctx, ro.ro_ctx_sync(ctx))
    want, after, n_used, pairs = compact(lists, refs)
    assert pages_out.tolist()[:len(want)] == want
    assert refs_out.tolist() == after.tolist() and used.item() == n_used and n_moves.item() == len(pairs)
    assert list(zip(t[0].tolist(), t[1].tolist()))[:len(pairs)] == pairs
    assert t[2].tolist()[:len(pairs)] == [page] * len(pairs)
    pool.check([(a, b, page) for a, b in pairs])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,used,page,layers", [(1, 0, 4, 1), (1, 1, 4, 1), (2, 1, 4, 1), (31, 17, 3, 1), (32, 32, 16, 1),
                                                (33, 1, 16, 2), (64, 0, 8, 1), (1000, 640, 4, 2), (20_000, 9_001, 1, 1),
                                                (5000, 4999, 2, 1), (70_001, 30_000, 1, 1)])
def test_compact(ctx, n, used, page, layers, in_place):
    g = np.random.default_rng(n + used)
    held = g.permutation(n)[:used].tolist()
    cuts = np.sort(g.integers(0, used + 1, 7))
    lists = [x.tolist() for x in np.split(np.asarray(held, np.int64), cuts)]
    refs = np.zeros(n, np.int64)
    for x in lists:
        for p in x:
            refs[p] += 1
    if used > 4:   # a shared prefix
        lists[0] = held[:3] + lists[0]
        refs[held[:3]] += 1
    run_compact(ctx, lists, refs, Pool(n, 2, page, 16, layers), page, in_place)


def test_compact_records_bad_entries(ctx):
    refs = np.array([0, 1, 0, 1, 0, 1])
    pool = Pool(6, 1, 4, 16)
    t, n = moves_of(3)
    for pages, want in (([1, 3, 99], [1, 0, 99]), ([1, 4, 5], [1, 4, 2]), ([1, 3, 2], [1, 0, 2])):
        out = torch.full((3,), -7, dtype=torch.int32, device="cuda")
        used = torch.zeros(1, dtype=torch.int32, device="cuda")
        ok(ctx, ro.ro_cache_compact(ctx, pool.caches(i64([0, 3]), i32(pages))[0], out, i32(refs), i32(refs), used,
                                    ro.ro_moves(*t, n)))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL and out.tolist() == want
    out = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    ok(ctx, ro.ro_cache_compact(ctx, pool.caches(i64([0, 3]), i32([1, 3, 5]))[0], out, i32(refs), i32(refs), used,
                                ro.ro_moves(*t, n)))
    assert ro.ro_ctx_sync(ctx) == ro.RO_E_CAPACITY and out.tolist() == [1, 0]


def test_copy_records_what_is_out_of_bounds(ctx):
    pool = Pool(8, 2, 16, 32)
    cache = pool.caches(i64([0, 1]), i32([0]))[0]
    for frm, to, slots, n, st, made in (([1, 9, 2], [5, 6, 7], [16, 16, 3], 3, ro.RO_E_INVAL, [(1, 5, 16), (2, 7, 3)]),
                                        ([1, 2, 3], [5, 60, 7], [16, 16, 17], 3, ro.RO_E_INVAL, [(1, 5, 16)]),
                                        ([1, 2, 3], [5, 6, 7], [0, 1, 15], 3, ro.RO_OK, [(2, 6, 1), (3, 7, 15)]),
                                        ([1, 2, 3], [5, 6, 7], [16, 1, 15], 9, ro.RO_E_CAPACITY, [(1, 5, 16), (2, 6, 1), (3, 7, 15)]),
                                        ([1, 2, 3], [5, 6, 7], [16, 1, 15], 0, ro.RO_OK, [])):
        pool = Pool(8, 2, 16, 32)
        cache = pool.caches(i64([0, 1]), i32([0]))[0]
        ok(ctx, ro.ro_cache_copy(ctx, cache, ro.ro_moves(i32(frm), i32(to), i32(slots), i32([n]))))
        assert ro.ro_ctx_sync(ctx) == st
        pool.check(made)


def test_offsets_past_32_bits(ctx):
    """A pool of 5 GB a side: the last page to the first, whole and in part."""
    k = torch.zeros(20_000, 16, 64, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[-1], v[-1], k[-2], v[-2] = 1, 2, 3, 4
    cache = ro.ro_cache(k, v, i64([0, 1]), i32([0]))
    ok(ctx, ro.ro_cache_copy(ctx, cache, ro.ro_moves(i32([19_999, 3]), i32([5, 19_998]), i32([64, 9]), i32([2]))))
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert bool((k[5] == 1).all()) and bool((v[5] == 2).all())
    assert bool((k[-2, :, :9] == 0).all()) and bool((v[-2, :, 9:] == 4).all()) and bool((k[-2, :, 9:] == 3).all())


def test_on_another_stream_and_in_a_graph(ctx):
    g = np.random.default_rng(1)
    lens = [100, 37, 64]
    lists, refs = some_lists(g, 80, lens, 16)
    side = torch.cuda.Stream()
    c2 = ro.ro_ctx_create(0, side, 1)
    try:
        kids, rooms = [2, 0, 3], [8, 7, 4, 5, 6]
        pool = Pool(80, 2, 16, 64)
        base, pages = i64(offsets([len(x) for x in lists])), i32([p for x in lists for p in x])
        cache = pool.caches(base, pages)[0]
        dst, len_out = torch.zeros(sum(rooms), dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
        refs_d = i32(refs)
        after = torch.zeros_like(refs_d)
        t, n = moves_of(40)
        args = (i32(lens), i64(offsets(kids)), i32([0, 0, 2, 2, 2]), i64(offsets(rooms)), i32(np.repeat(range(5), rooms)))
        moves = ro.ro_moves(*t, n)
        out2, after2, used = torch.zeros_like(pages), torch.zeros_like(refs_d), torch.zeros(1, dtype=torch.int32, device="cuda")

        def both():
            ok(c2, ro.ro_cache_fork(c2, cache, *args, dst, len_out, refs_d, after, moves))
            ok(c2, ro.ro_cache_compact(c2, cache, out2, refs_d, after2, used, moves))

        torch.cuda.synchronize()
        both()
        ok(c2, ro.ro_ctx_sync(c2))
        new, want_len, want_after, _, _ = fork(lists, lens, kids, rooms, refs, 16)
        want2, want_after2, want_used, _ = compact(lists, refs)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both()
        for _ in range(2):
            for x in (dst, len_out, after, out2, after2, used):
                x.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.synchronize()
            assert dst.tolist() == [p for x in new for p in x] and after.tolist() == want_after.tolist()
            assert len_out.tolist() == want_len and out2.tolist() == want2
            assert after2.tolist() == want_after2.tolist() and used.item() == want_used
        ok(c2, ro.ro_ctx_sync(c2))
    finally:
        ro.ro_ctx_destroy(c2)


def test_refusals(ctx):
    pool = Pool(8, 1, 16, 32)
    base, pages, refs = i64([0, 2]), i32([1, 3]), i32([0, 1, 0, 1, 0, 0, 0, 0])
    cache = pool.caches(base, pages)[0]
    t, n = moves_of(4)
    moves = ro.ro_moves(*t, n)
    lens, after = i32([20]), torch.zeros_like(refs)

    def status(**change):
        a = dict(cache=cache, d_len=lens, d_child_base=i64([0, 1]), d_child_parent=i32([0]), d_dst_base=i64([0, 2]),
                 d_dst_seq=i32([0, 0]), d_dst_pages=torch.zeros(2, dtype=torch.int32, device="cuda"),
                 d_len_out=torch.zeros(1, dtype=torch.int32, device="cuda"), d_refs=refs, d_refs_out=after, moves=moves)
        a.update(change)
        return ro.ro_cache_fork(ctx, *a.values())

    assert status(d_len_out=lens) == ro.RO_E_INVAL
    assert status(d_dst_pages=pages) == ro.RO_E_INVAL
    both = torch.zeros(16, dtype=torch.int32, device="cuda")
    assert status(d_refs=both[:8], d_refs_out=both[4:12]) == ro.RO_E_INVAL
    for bad in (dict(d_refs=refs[:7].clone()), dict(d_refs_out=after[:7].clone()), dict(d_dst_base=i64([0])),
                dict(d_child_base=i64([0])), dict(d_dst_pages=i32([0])), dict(d_len=i32([])),
                dict(moves=ro.ro_moves(t[0][:0], t[1][:0], t[2][:0], n))):
        with pytest.raises(ValueError):
            status(**bad)
    with pytest.raises(ValueError):
        ro.ro_cache_compact(ctx, cache, pages, refs, after, n, ro.ro_moves(t[0][:3], t[1][:3], t[2][:3], n))
    assert ro.ro_cache_compact(ctx, cache, pages, both[:8], both[4:12], n, moves) == ro.RO_E_INVAL
    ok(ctx, ro.ro_ctx_sync(ctx))
    ok(ctx, status())
    ok(ctx, ro.ro_ctx_sync(ctx))


def test_outputs_that_share_memory_are_refused(ctx):
    """An output on an input or on another output, in part or in whole, where the header does not allow it."""
    pool = Pool(8, 1, 16, 32)
    base, pages, refs = i64([0, 2]), i32([1, 3]), i32([0, 1, 0, 1, 0, 0, 0, 0])
    cache = pool.caches(base, pages)[0]
    t, n = moves_of(8)
    moves = ro.ro_moves(*t, n)
    free = torch.zeros(64, dtype=torch.int32, device="cuda")
    good = dict(cache=cache, d_len=i32([20]), d_child_base=i64([0, 1]), d_child_parent=i32([0]), d_dst_base=i64([0, 2]),
                d_dst_seq=i32([0, 0]), d_dst_pages=free[:2], d_len_out=free[8:9], d_refs=refs, d_refs_out=free[16:24], moves=moves)

    def fork(**change):
        return ro.ro_cache_fork(ctx, *{**good, **change}.values())

    for bad in (dict(d_dst_pages=good["d_dst_seq"]), dict(d_len_out=good["d_child_parent"]), dict(d_dst_pages=free[17:19]),
                dict(d_len_out=free[1:2]), dict(d_dst_pages=t[1][:2]), dict(d_refs_out=t[0]), dict(d_len_out=n),
                dict(d_dst_pages=refs[:2]), dict(moves=ro.ro_moves(t[0], t[0], t[2], n)),
                dict(moves=ro.ro_moves(t[0], t[1], t[2], t[2][:1])), dict(moves=ro.ro_moves(t[0], refs, t[2], n))):
        assert fork(**bad) == ro.RO_E_INVAL, bad
    used = free[32:33]

    def compact(out=free[:2], counts=free[16:24], used=used, m=moves):
        return ro.ro_cache_compact(ctx, cache, out, refs, counts, used, m)

    for bad in (dict(out=free[16:18]), dict(out=refs[:2]), dict(counts=t[2]), dict(used=n), dict(used=refs[:1]),
                dict(used=free[1:2]), dict(m=ro.ro_moves(t[0], t[1], t[1], n))):
        assert compact(**bad) == ro.RO_E_INVAL, bad
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert not free.any() and refs.tolist() == [0, 1, 0, 1, 0, 0, 0, 0]
    ok(ctx, fork())
    ok(ctx, compact())
    ok(ctx, fork(d_refs=free[16:24].copy_(refs), d_refs_out=free[16:24]))   # in place
    ok(ctx, ro.ro_ctx_sync(ctx))
