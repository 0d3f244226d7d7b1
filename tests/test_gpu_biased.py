"""Attention with capped scores, distance biases, document and prefix masks on
the GPU against its definition in 64 bits: every kernel's sizes, masks that
leave rows empty, contents that must not be used, splits, strides, streams."""
import math

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
from tests import bias_reference as ref  # noqa: E402
from tests.step_reference import Cache  # noqa: E402

BF16, F16 = torch.bfloat16, torch.float16
NOTHING = 2 ** 31 - 1


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


def starts(news):
    return np.concatenate([[0], np.cumsum(news)])


def within(got, want, tol):
    got = got.double().cpu()
    assert not torch.isnan(got).any()
    bad = (got - want).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst by {float(((got - want).abs() - tol).max()):.3g}"


def masks(lens, news, docs, frame, seed, pads=0.1):
    """Each token's first slot (documents of about `docs` tokens, some tokens padding) and its frame's end."""
    g = np.random.default_rng(seed)
    first, until = [], []
    for L, n in zip(lens, news):
        a = np.arange(L - n, L)
        if docs:
            cuts = np.concatenate([[0], np.cumsum(g.integers(1, 2 * docs + 1, 2 * max(L, 1) // docs + 8))])
            f = cuts[np.searchsorted(cuts, np.maximum(a, 0), side="right") - 1]
            first.append(np.where(g.random(n) < pads, NOTHING, f))
        if frame:
            until.append((np.maximum(a, 0) // frame + 1) * frame)   # past the end of the cache, too
    return (np.concatenate(first) if docs else None), (np.concatenate(until) if frame else None)


class Case:
    def __init__(self, c, news, heads, window=0, sinks=0, cap=0.0, slopes=False, first=None, until=None, scale=None, seed=0):
        self.c, self.news, self.heads, self.window, self.sinks, self.cap = c, news, heads, window, sinks, cap
        dt, dim = c.k.dtype, c.k.shape[3]
        self.scale = 1 / math.sqrt(dim) if scale is None else scale
        g = torch.Generator().manual_seed(seed)
        self.q = torch.randn(sum(news), heads + 1, dim, generator=g).to(dt)[:, :heads]
        self.slope = 2.0 ** (-8.0 * torch.arange(1, heads + 1) / heads) if slopes else None
        self.first = None if first is None else torch.as_tensor(np.asarray(first, np.int64))
        self.until = None if until is None else torch.as_tensor(np.asarray(until, np.int64))

    def device(self):
        self.dq = torch.zeros(self.q.shape[0], self.heads + 1, self.q.shape[2], dtype=self.q.dtype, device="cuda")[:, :self.heads]
        self.dq.copy_(self.q)
        self.cache = ro.ro_cache(self.c.k.cuda(), self.c.v.cuda(), i64(self.c.base), self.c.pages.cuda())
        self.bias = ro.ro_bias(self.cap, None if self.slope is None else self.slope.float().cuda(),
                               None if self.first is None else i32(self.first),
                               None if self.until is None else i32(self.until))
        self.tok_base, self.len = i64(starts(self.news)), i32(self.c.lens)
        self.out = torch.full_like(self.dq, 9.0).contiguous()
        self.lse = torch.full(self.q.shape[:2], 9.0, device="cuda")
        return self

    def call(self, ctx, max_len=None, max_new=None):
        ok(ctx, ro.ro_cache_attend_biased(ctx, self.cache, self.tok_base, max(self.news) if max_new is None else max_new,
                                          self.len, max(self.c.lens) if max_len is None else max_len, self.dq, self.scale,
                                          self.window, self.sinks, self.bias, self.out, self.lse))

    def check(self, ctx, **kw):
        self.device().call(ctx, **kw)
        ok(ctx, ro.ro_ctx_sync(ctx))
        t = starts(self.news)
        for s, n in enumerate(self.news):
            if n == 0:
                continue
            r = slice(t[s], t[s + 1])
            out, lse, tol, lse_tol = ref.attend(self.c, s, self.q[r], self.scale, self.window, self.sinks, self.cap,
                                                self.slope, None if self.first is None else self.first[r],
                                                None if self.until is None else self.until[r])
            within(self.out[r], out, tol)
            got, empty = self.lse[r].double().cpu(), torch.isinf(lse)
            assert torch.equal(torch.isinf(got) & (got < 0), empty)
            within(got[~empty], lse[~empty], lse_tol[~empty])
        return self.out, self.lse


FORMS = [dict(cap=30.0), dict(cap=0.5), dict(slopes=True), dict(docs=40), dict(frame=50), dict(docs=30, frame=9),
         dict(cap=5.0, slopes=True, docs=60, frame=25), dict(window=20, sinks=3, docs=50),
         dict(window=70, sinks=66, frame=33, cap=2.0), dict(window=1, slopes=True)]


def build(lens, news, kv, dim, page, dtype, heads, form, seed, pads=0.1, **kw):
    f = dict(form)
    first, until = masks(lens, news, f.pop("docs", 0), f.pop("frame", 0), seed, pads)
    return Case(Cache(lens, kv, dim, page, dtype, seed, **kw), news, heads, first=first, until=until, seed=seed, **f)


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("dtype,dim,heads,kv,page", [(BF16, 128, 4, 2, 64), (F16, 64, 2, 2, 16), (BF16, 80, 6, 2, 5),
                                                     (F16, 128, 3, 1, 20), (F16, 96, 130, 1, 16), (BF16, 40, 8, 1, 256)])
def test_chunks(ctx, dtype, dim, heads, kv, page, form):
    news = [33, 1, 0, 70, 129] if heads < 100 else [3, 1, 0, 2, 5]
    lens = [33, 200, 50, 131, 300]
    build(lens, news, kv, dim, page, dtype, heads, FORMS[form], page + form).check(ctx)


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("dtype,dim,heads,kv,page", [(BF16, 128, 8, 1, 64), (F16, 64, 4, 2, 16), (BF16, 80, 3, 3, 5),
                                                     (F16, 8, 7, 1, 128), (BF16, 96, 4, 4, 32)])
@pytest.mark.parametrize("news", [[1, 1, 1, 1, 0, 1], [1, 2, 2, 1, 0, 2]])
def test_few_rows(ctx, dtype, dim, heads, kv, page, news, form):
    lens = [1, 64, 65, 300, 0, 777]
    build(lens, news, kv, dim, page, dtype, heads, FORMS[form], form).check(ctx)


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("dtype,dim,page", [(BF16, 128, 64), (F16, 64, 4), (BF16, 80, 5)])
def test_many_short_sequences(ctx, dtype, dim, page, form):
    g = np.random.default_rng(form)
    lens = [int(x) for x in g.integers(0, 140, 260)]
    lens[:6] = [0, 1, 16, 17, 32, 139]
    news = [min(L, int(x)) for L, x in zip(lens, g.integers(0, 5, 260))]
    case = build(lens, news, 4, dim, page, dtype, 8, FORMS[form], form)
    out, lse = case.check(ctx, max_len=139)
    again, lse2 = case.check(ctx, max_len=139)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("news,lens", [([60, 9], [300, 40]), ([2, 1], [300, 40]), ([1, 1], [1, 300])])
@pytest.mark.parametrize("page", [16, 7])
def test_unseen_slots_are_never_used(ctx, junk, news, lens, page):
    """Whatever lies in other documents, behind windows and frames, and in the slots of tokens that only pad."""
    for form in (dict(docs=12), dict(docs=12, frame=5), dict(docs=40, window=6, sinks=2), dict(window=9, sinks=3, frame=4)):
        case = build(lens, news, 2, 64, page, BF16, 4, form, 3, pads=0.3)
        t = starts(news)
        for s, n in enumerate(news):
            first = None if case.first is None else case.first[t[s]:t[s + 1]]
            until = None if case.until is None else case.until[t[s]:t[s + 1]]
            m = ref.seen(lens[s], n, case.window, case.sinks, first, until).any(0)
            for j in np.flatnonzero(~m.numpy()):
                at = int(case.c.pages[case.c.base[s] + j // page])
                case.c.k[at, :, j % page] = junk
                case.c.v[at, :, j % page] = junk
        case.check(ctx)


def test_documents_in_no_order(ctx):
    """First slots that rise and fall from token to token, with a window and sinks, junk wherever nobody looks."""
    g = np.random.default_rng(5)
    for news in ([90, 40], [2, 2]):
        lens = [400, 70]
        c = Cache(lens, 2, 64, 16, F16, 1)
        first = np.concatenate([g.integers(0, L, n) for L, n in zip(lens, news)])
        case = Case(c, news, 4, 11, 4, first=first, slopes=True)
        t = starts(news)
        for s, n in enumerate(news):
            m = ref.seen(lens[s], n, 11, 4, case.first[t[s]:t[s + 1]]).any(0)
            for j in np.flatnonzero(~m.numpy()):
                at = int(c.pages[c.base[s] + j // 16])
                c.k[at, :, j % 16] = float("nan")
                c.v[at, :, j % 16] = float("nan")
        case.check(ctx)


@pytest.mark.parametrize("news", [[5, 40], [1, 1], [2, 3]])
def test_rows_that_see_nothing(ctx, news):
    """Padding alone, a chunk longer than its cache, a document that starts behind its token."""
    lens = [3, 50]
    c = Cache(lens, 2, 64, 16, BF16, 2)
    case = Case(c, news, 4, first=[NOTHING] * sum(news))
    out, lse = case.check(ctx)
    assert bool((out == 0).all()) and bool(torch.isinf(lse).all())
    Case(c, news, 4, first=[1] * news[0] + [49] * news[1], cap=3.0).check(ctx)
    Case(c, [9, 1], 4, cap=3.0, slopes=True, until=[7] * 10).check(ctx)


@pytest.mark.parametrize("cap", [1e-6, 1e-3, 1.0, 40.0, 69.0, 75.0, 1e4, 1e30])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news", [[1, 2], [90, 60]])
@pytest.mark.parametrize("scale", [0.125, -0.5, 0.0, 6.0])
def test_caps_and_scales(ctx, cap, news, scale, dtype):
    Case(Cache([500, 90], 2, 64, 32, dtype, 8), news, 4, cap=cap, scale=scale, slopes=cap == 40.0).check(ctx)


@pytest.mark.parametrize("news", [[1, 2], [90, 60]])
def test_infinite_scores_under_a_cap(ctx, news):
    """Products past 32 bits' range are the cap, on either side."""
    c = Cache([130, 90], 2, 64, 32, BF16, 8)
    big = 2.0 ** 127
    for s, j in ((0, 3), (1, 5)):
        c.k[int(c.pages[c.base[s]]), :, j] = big
    case = Case(c, news, 4, cap=8.0)
    case.q[:] = case.q.abs() + 4.0    # 64 products of 2^129: infinite
    case.q[::2] *= -1
    case.check(ctx)


@pytest.mark.parametrize("form", [0, 2, 4, 6, 8])
@pytest.mark.parametrize("news", [[2, 3], [70, 20], [700, 3]])
@pytest.mark.parametrize("page", [64, 7])
def test_long_caches_split_and_join(ctx, news, form, page):
    case = build([9000, 700], news, 1, 64, page, BF16, 4, FORMS[form], 4)
    if form == 4:
        case.until[:news[0]] = 9000      # a prefix
    out, lse = case.check(ctx)
    for max_len in (0, 100, 1 << 30):
        case.check(ctx, max_len=max_len)
    again, lse2 = case.check(ctx)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("window,sinks", [(2 ** 32 - 1, 0), (2 ** 31, 5), (3, 2 ** 32 - 1), (70, 2 ** 31)])
@pytest.mark.parametrize("news", [[1, 1], [50, 90]])
def test_windows_past_every_slot(ctx, news, window, sinks):
    case = build([200, 300], news, 2, 64, 16, BF16, 4, dict(docs=60, cap=9.0, window=window, sinks=sinks), 7)
    case.check(ctx)


def test_without_a_bias_it_is_plain_attention(ctx):
    for news in ([1, 1], [60, 130]):
        c = Cache([300, 200], 2, 128, 64, BF16, 9)
        case = Case(c, news, 8)
        out, lse = case.check(ctx)
        plain, plain_lse = torch.zeros_like(out), torch.zeros_like(lse)
        ok(ctx, ro.ro_cache_attend(ctx, case.cache, case.tok_base, max(news), case.len, 300, case.dq, case.scale, 0, 0, plain,
                                   plain_lse))
        ok(ctx, ro.ro_ctx_sync(ctx))
        # two roundings of one value: a step apart at most, and what the tile's weights may differ by
        assert float((out.float() - plain.float()).abs().max()) <= 2 * 2.0 ** -8 * 4
        assert float((lse - plain_lse).abs().max()) <= 1e-5


def test_offsets_past_32_bits(ctx):
    """Pages whose elements lie past 2^32: a pool of 9 GB."""
    n, page, heads, dim = 40_000, 64, 14, 128
    k = torch.zeros(n, heads, page, dim, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    pages = [n - 1, 3, n - 2, 39_000]
    g = torch.Generator().manual_seed(1)
    c = Cache([200, 55], heads, dim, page, BF16, 3, junk=0.0)
    for s, L in enumerate(c.lens):
        for i in range(-(-L // page)):
            at = int(c.pages[c.base[s] + i])
            to = pages.pop() if pages else 38_000 - i
            k[to], v[to] = c.k[at].cuda(), c.v[at].cuda()
            c.pages[c.base[s] + i] = to | (at << 20)   # both, unpacked below
    to, at = c.pages & 0xFFFFF, c.pages >> 20
    for news in ([1, 1], [60, 55]):
        c.pages = at.int()
        case = Case(c, news, heads, cap=20.0, first=[0] * sum(news), seed=int(torch.randint(9, (1,), generator=g)))
        case.device()
        case.cache = ro.ro_cache(k, v, i64(c.base), to.int().cuda())
        case.call(ctx)
        ok(ctx, ro.ro_ctx_sync(ctx))
        t = starts(news)
        for s in range(2):
            r = slice(t[s], t[s + 1])
            out, lse, tol, lse_tol = ref.attend(c, s, case.q[r], case.scale, 0, 0, 20.0, None, case.first[r])
            within(case.out[r], out, tol)
            within(case.lse[r], lse, lse_tol)


def test_bad_pages_and_ranges_are_recorded(ctx):
    for news in ([1, 1], [40, 70]):
        lens = [100, 90]
        c = Cache(lens, 2, 64, 16, BF16, 3, junk=0.0)
        case = Case(c, news, 4, cap=5.0, first=[0] * sum(news)).device()
        case.call(ctx)
        ok(ctx, ro.ro_ctx_sync(ctx))
        good = case.out.clone()
        bad = c.pages.clone()
        bad[0] = 60_000
        case.cache = ro.ro_cache(c.k.cuda(), c.v.cuda(), i64(c.base), bad.cuda())
        case.call(ctx)
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
        assert torch.equal(case.out[news[0]:], good[news[0]:])
        case.cache = ro.ro_cache(c.k.cuda(), c.v.cuda(), i64(c.base), c.pages.cuda())
        case.len = i32([1000, 90])
        case.call(ctx)
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_CAPACITY
        case.len = i32(lens)
        case.tok_base = i64([0, news[0], 10_000])
        case.call(ctx, max_new=20_000)
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
        case.tok_base = i64(starts(news))
        case.call(ctx)
        ok(ctx, ro.ro_ctx_sync(ctx))
        assert torch.equal(case.out, good)


def test_on_another_stream_and_in_a_graph(ctx):
    side = torch.cuda.Stream()
    c2 = ro.ro_ctx_create(0, side, 1)
    try:
        for news in ([1, 1], [80, 140], [3, 300]):
            case = build([4000, 500], news, 2, 64, 16, BF16, 4, FORMS[6], 11)
            want, want_lse = [x.clone() for x in case.check(ctx)]
            torch.cuda.synchronize()
            case.call(c2)
            ok(c2, ro.ro_ctx_sync(c2))
            assert torch.equal(case.out, want)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                case.call(c2)
            for _ in range(3):
                case.out.zero_()
                case.lse.zero_()
                torch.cuda.synchronize()
                with torch.cuda.stream(side):
                    graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(case.out, want) and torch.equal(case.lse, want_lse)
            ok(c2, ro.ro_ctx_sync(c2))
    finally:
        ro.ro_ctx_destroy(c2)


def test_refusals(ctx):
    case = Case(Cache([20], 2, 64, 16, BF16, 1), [3], 4, cap=5.0).device()

    def status(**change):
        a = dict(cache=case.cache, d_tok_base=case.tok_base, max_new=3, d_len=case.len, max_len=20, d_q=case.dq, scale=0.1,
                 window=0, sinks=0, bias=case.bias, d_out=case.out, d_lse=case.lse)
        a.update(change)
        return ro.ro_cache_attend_biased(ctx, *a.values())

    before = case.out.clone()
    for cap in (-1.0, math.nan, math.inf, 1e-7):
        assert status(bias=ro.ro_bias(cap)) == ro.RO_E_INVAL
    assert status(bias=ro.ro_bias(1e-6), scale=1e30) == ro.RO_E_INVAL
    assert status(scale=math.inf) == ro.RO_E_INVAL
    assert status(d_out=case.dq) == ro.RO_E_INVAL
    for bad in (dict(d_slope=torch.zeros(3, device="cuda")), dict(d_first=torch.zeros(2, dtype=torch.int32, device="cuda")),
                dict(d_until=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            status(bias=ro.ro_bias(1.0, **bad))
    assert status(bias=ro.ro_bias(1.0, d_first=case.len.data_ptr() + 2)) == ro.RO_E_INVAL
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert torch.equal(case.out, before)
    ok(ctx, status())
    ok(ctx, ro.ro_ctx_sync(ctx))


@pytest.mark.parametrize("cap", [5.0, 30.0, 50.0, 75.0])
@pytest.mark.parametrize("size", [2.0 ** 60, 2.0 ** 30, 2.0 ** -30])
@pytest.mark.parametrize("sign", [1, -1])
def test_values_of_any_size_under_a_cap(ctx, cap, size, sign):
    """Scores near the cap on either side, values far from 1."""
    c = Cache([400, 90], 2, 64, 32, BF16, 8)
    c.v[:] = (c.v.double() * size).to(BF16)
    case = Case(c, [90, 60], 4, cap=cap, scale=0.125)
    case.q[:] = case.q.abs() * 4
    c.k[:] = (c.k.abs() + 2) * sign      # products far beyond the cap
    case.check(ctx)
