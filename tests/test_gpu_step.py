"""The model-step operators on the GPU against their definitions in 64 bits:
rotary positions and their gradient, the paged cache's append, attention,
weights and eviction, at the sizes, masks, strides and contents where they can
go wrong, with what they refuse and what they record."""
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
from tests import step_reference as ref  # noqa: E402

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture
def ctx():
    c = ro.ro_ctx_create(0, torch.cuda.current_stream(), 1)
    yield c
    ro.ro_ctx_destroy(c)


def ok(ctx, status):
    assert status == ro.RO_OK, ro.ro_last_error(ctx)


def sync_ok(ctx):
    ok(ctx, ro.ro_ctx_sync(ctx))


def i64(x):
    return torch.as_tensor(np.asarray(x, np.int64)).cuda()


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def within(got, want, tol):
    got = got.double().cpu()
    assert not torch.isnan(got).any()
    bad = (got - want).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst by {float(((got - want).abs() - tol).max()):.3g}"


def starts(news):
    return np.concatenate([[0], np.cumsum(news)])


def token_seq(news):
    return i32(np.repeat(np.arange(len(news)), news))


def on_gpu(cache):
    k, v = cache.k.cuda(), cache.v.cuda()
    return ro.ro_cache(k, v, i64(cache.base), cache.pages.cuda()), k, v


# ---------------------------------------------------------------------------- rotary
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("dim,pairs", [(128, [32, 16, 16]), (80, [40]), (40, [8, 6, 6]), (64, [4, 3]), (2, [1]),
                                       (256, [32, 32, 32, 32]), (18, [9]), (30, [2, 1, 3, 2])])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(ctx, dtype, dim, pairs, interleaved):
    g = torch.Generator().manual_seed(dim + interleaved)
    T, H = 37, 5
    x = torch.randn(T, H, dim, generator=g).to(dtype)
    pos = torch.randint(-1000, 100_000, (T, len(pairs)), generator=g, dtype=torch.int32)
    pos[:2] = torch.tensor([[0], [2 ** 31 - 1]], dtype=torch.int32)
    rope = ro.ro_rope(pairs, base=10_000.0, interleaved=interleaved)
    for inverse in (False, True):
        out = torch.zeros(T, H, dim, dtype=dtype, device="cuda")
        ok(ctx, ro.ro_rotary(ctx, x.cuda(), out, pos.cuda(), rope, inverse))
        sync_ok(ctx)
        want = ref.turn(x, pos, pairs, 10_000.0, interleaved, inverse)
        # angle: 2^-24 of half a turn and 1e-6 of a radian for the largest position; two products, one sum
        size = ref.turn(x.abs(), pos * 0, pairs, 10_000.0, interleaved).abs()
        partner = want.abs() + x.double().abs().amax(-1, keepdim=True)
        within(out, want, (math.pi * 2.0 ** -24 + 1.2e-6 + 3 * 2.0 ** -24) * (size + partner) + ref.U[dtype] * want.abs()
               + ref.TINY[dtype])


def test_rotary_strides_in_place_and_odd_alignment(ctx):
    rope = ro.ro_rope([4, 4], base=100.0)
    pos = torch.randint(0, 50, (9, 2), dtype=torch.int32)
    for offset, width in [(0, 24), (1, 23), (3, 26)]:
        fused = torch.randn(9 * 3 * width + 8, dtype=F32).to(BF16)
        view = fused[offset:offset + 9 * 3 * width].view(9, 3, width)[..., :20]
        want = ref.turn(view, pos, [4, 4], 100.0, False)
        dev = fused.cuda()
        x = dev[offset:offset + 9 * 3 * width].view(9, 3, width)[..., :20]
        ok(ctx, ro.ro_rotary(ctx, x, x, pos.cuda(), rope))
        sync_ok(ctx)
        within(x, want, ref.U[BF16] * want.abs() + 1e-5)
        rest = torch.ones(fused.numel(), dtype=torch.bool)
        rest[offset:offset + 9 * 3 * width].view(9, 3, width)[..., :20] = False
        assert torch.equal(dev.cpu()[rest], fused[rest])   # nothing beside the view changed


def test_rotary_gradient(ctx):
    """inverse is the gradient: against the formula's (autograd in 64 bits) and against differences."""
    T, H, D, pairs = 5, 2, 12, [2, 3]
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(0, 4000, (T, 2), generator=g, dtype=torch.int32)
    x = torch.randn(T, H, D, generator=g, dtype=torch.float64)
    w = torch.randn(T, H, D, generator=g)
    rope = ro.ro_rope(pairs)
    grad = torch.zeros(T, H, D, device="cuda")
    ok(ctx, ro.ro_rotary(ctx, w.cuda(), grad, pos.cuda(), rope, True))
    sync_ok(ctx)
    R = sum(pairs)
    axis = torch.repeat_interleave(torch.arange(2), torch.tensor(pairs))
    theta = pos[:, axis].double() * 10_000.0 ** (-torch.arange(R).double() / R)
    z = x.clone().requires_grad_()
    a, b = z[..., :R], z[..., R:2 * R]
    c, s = theta.cos()[:, None], theta.sin()[:, None]
    (torch.cat([a * c - b * s, b * c + a * s, z[..., 2 * R:]], -1) * w.double()).sum().backward()
    within(grad, z.grad, 1e-6 * (1 + w.double().abs().amax(-1, keepdim=True)))

    def value(v):
        out = torch.zeros(T, H, D, device="cuda")
        ok(ctx, ro.ro_rotary(ctx, v.float().cuda(), out, pos.cuda(), rope))
        sync_ok(ctx)
        return float((out.double().cpu() * w.double()).sum())

    x = x.float().double()
    for _ in range(6):
        d = torch.randn(T, H, D, generator=g).double()
        slope = (value(x + 0.5 * d) - value(x - 0.5 * d))
        # the turn is linear: the difference is exact but for 32-bit rounding of its 240 terms
        assert abs(slope - float((grad.double().cpu() * d).sum())) < 240 * 8 * 2.0 ** -22 * 4


# ---------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page,dim,heads,kv", [(16, 64, 4, 2), (3, 40, 5, 5), (64, 128, 6, 1), (1, 8, 2, 2)])
def test_append(ctx, dtype, page, dim, heads, kv):
    lens, news = [70, 1, 0, 33, 129], [17, 1, 0, 33, 0]
    c = ref.Cache(lens, kv, dim, page, dtype, 5, junk=7.0)
    T = sum(news)
    g = torch.Generator().manual_seed(page)
    fused = torch.randn(T, heads + 2 * kv, dim, generator=g).to(dtype)
    pairs = [dim // 2 - dim // 4, dim // 4]
    pos = torch.randint(0, 3000, (T, 2), generator=g, dtype=torch.int32)
    cache, k, v = on_gpu(c)
    dev = fused.cuda()
    q_out = torch.zeros(T, heads, dim, dtype=dtype, device="cuda")
    for rope in (ro.ro_rope(pairs), None):
        ok(ctx, ro.ro_cache_append(ctx, cache, i64(starts(news)), token_seq(news), i32(lens), pos.cuda(), rope,
                                   dev[:, :heads], q_out, dev[:, heads:heads + kv], dev[:, heads + kv:]))
        sync_ok(ctx)
        turned = ref.turn(fused, pos, pairs, 10_000.0, False) if rope else fused.double()
        tol = (ref.U[dtype] * turned.abs() + 1e-5) if rope else turned * 0
        within(q_out, turned[:, :heads], tol[:, :heads])
        want_k, want_v = c.k.double(), c.v.double()
        tol_k = torch.zeros_like(want_k)
        for s, (L, n) in enumerate(zip(lens, news)):
            for i in range(n):
                j, t = L - n + i, starts(news)[s] + i
                at = int(c.pages[c.base[s] + j // page])
                want_k[at, :, j % page], want_v[at, :, j % page] = turned[t, heads:heads + kv], fused[t, heads + kv:].double()
                tol_k[at, :, j % page] = tol[t, heads:heads + kv]
        within(k, want_k, tol_k)
        assert torch.equal(v.double().cpu(), want_v)


def test_append_leaves_out_what_does_not_fit(ctx):
    """A chunk longer than its cache, too few pages, a bad page, a bad sequence: recorded or left out, nothing else written."""
    c = ref.Cache([8, 8], 1, 8, 4, BF16, 1, spare=2, junk=0.0)
    x = torch.ones(6, 1, 8, dtype=BF16, device="cuda")

    def call(base, pages, tok_base, seq, lens):
        k, v = torch.zeros_like(c.k).cuda(), torch.zeros_like(c.v).cuda()
        cache = ro.ro_cache(k, v, i64(base), i32(pages))
        ok(ctx, ro.ro_cache_append(ctx, cache, i64(tok_base), i32(seq), i32(lens), None, None, None, None, x, x))
        return ro.ro_ctx_sync(ctx), k[:, 0, :, 0].float().cpu().numpy()

    st, k = call([0, 2, 4], [5, 0, 1, 2], [0, 3, 6], [0] * 3 + [1] * 3, [1, 8])
    assert st == ro.RO_OK and k.sum() == 1 + 3 and k[5, 0] == 1 and list(k[2]) == [0, 1, 1, 1]
    st, k = call([0, 2, 4], [5, 0, 1, 2], [0, 3, 6], [0] * 3 + [1] * 3, [10, 8])
    assert st == ro.RO_E_CAPACITY and list(k[0]) == [0, 0, 0, 1]
    st, k = call([0, 2, 4], [5, 6, 1, 2], [0, 3, 6], [0] * 3 + [1] * 3, [6, 8])
    assert st == ro.RO_E_INVAL and k.sum() == 1 + 3
    st, k = call([0, 2, 4], [5, 0, 1, 2], [0, 3, 6], [0] * 3 + [2] * 3, [6, 8])
    assert st == ro.RO_E_INVAL and k.sum() == 3
    sync_ok(ctx)   # reported once


# ---------------------------------------------------------------------------- attend
def run_attend(ctx, c, news, heads, scale, window, sinks, seed=0, max_len=None, max_new=None, gpu=None):
    dt, kv, dim = c.k.dtype, c.k.shape[1], c.k.shape[3]
    T = sum(news)
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(T, heads + 1, dim, generator=g).to(dt)
    cache, _, _ = gpu or on_gpu(c)
    out = torch.full((T, heads, dim), 9.0, dtype=dt, device="cuda")
    lse = torch.full((T, heads), 9.0, device="cuda")
    dq = q.cuda()
    ok(ctx, ro.ro_cache_attend(ctx, cache, i64(starts(news)), max(news) if max_new is None else max_new, i32(c.lens),
                               max(c.lens) if max_len is None else max_len, dq[:, :heads], scale, window, sinks, out, lse))
    sync_ok(ctx)
    return q[:, :heads], dq[:, :heads], out, lse


def check_attend(ctx, c, news, heads, window=0, sinks=0, scale=None, **kw):
    scale = 1 / math.sqrt(c.k.shape[3]) if scale is None else scale
    q, _, out, lse = run_attend(ctx, c, news, heads, scale, window, sinks, **kw)
    t = starts(news)
    for s in range(len(news)):
        if news[s] == 0:
            continue
        w_out, w_lse, tol, lse_tol = ref.attend(c, s, q[t[s]:t[s + 1]], scale, window, sinks)
        within(out[t[s]:t[s + 1]], w_out, tol)
        empty = torch.isinf(w_lse)
        got = lse[t[s]:t[s + 1]].double().cpu()
        assert torch.equal(torch.isinf(got) & (got < 0), empty)
        within(got[~empty], w_lse[~empty], lse_tol[~empty])
    return out, lse


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,heads,kv", [(64, 4, 2), (128, 8, 1), (80, 3, 3), (96, 5, 1), (8, 7, 1), (40, 20, 1)])
@pytest.mark.parametrize("page", [16, 5, 128])
def test_attend_single_tokens(ctx, dtype, dim, heads, kv, page):
    lens = [1, 64, 65, 300, 0, 777]
    check_attend(ctx, ref.Cache(lens, kv, dim, page, dtype, dim), [1, 1, 1, 1, 0, 1], heads)


@pytest.mark.parametrize("dtype,dim,heads,kv,page", [(BF16, 128, 4, 2, 64), (F16, 64, 2, 2, 16), (BF16, 80, 6, 2, 32),
                                                     (F16, 128, 3, 1, 20), (BF16, 64, 7, 1, 128), (BF16, 128, 2, 1, 8),
                                                     (F16, 96, 130, 1, 16), (BF16, 40, 8, 1, 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (7, 3), (64, 4), (130, 70)])
def test_attend_chunks(ctx, dtype, dim, heads, kv, page, window, sinks):
    """Ragged chunks over ragged caches: whole prompts, one token, none, chunk edges inside pages and tiles."""
    news = [33, 1, 0, 70, 129] if heads < 100 else [3, 1, 0, 2, 5]
    lens = [33, 200, 50, 131, 300]
    check_attend(ctx, ref.Cache(lens, kv, dim, page, dtype, page), news, heads, window, sinks)


@pytest.mark.parametrize("dtype,dim,heads,kv,page", [(BF16, 128, 8, 4, 64), (F16, 64, 4, 4, 16), (BF16, 80, 12, 4, 4),
                                                     (F16, 40, 4, 4, 20), (BF16, 96, 4, 4, 5), (F16, 128, 4, 4, 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 2), (40, 35)])
def test_attend_many_short_sequences(ctx, dtype, dim, heads, kv, page, window, sinks):
    """More sequences and heads than the GPU holds at once: empty ones, one token, ends inside stages and pages."""
    g = np.random.default_rng(dim + page + window)
    lens = [int(x) for x in g.integers(0, 140, 260)]
    lens[:6] = [0, 1, 16, 17, 32, 139]
    news = [min(L, int(x)) for L, x in zip(lens, g.integers(0, 5, 260))]
    c = ref.Cache(lens, kv, dim, page, dtype, 50)
    out, lse = check_attend(ctx, c, news, heads, window, sinks, max_len=139)
    again = run_attend(ctx, c, news, heads, 1 / math.sqrt(dim), window, sinks, max_len=139)
    assert torch.equal(out, again[2]) and torch.equal(lse, again[3])


def test_attend_short_sequences_bad_pages_and_lengths_are_recorded(ctx):
    lens = [40] * 400
    c = ref.Cache(lens, 2, 64, 16, BF16, 3, junk=0.0)
    good = run_attend(ctx, c, [1] * 400, 2, 0.1, 0, 0)
    cache, _, _ = on_gpu(c)
    out = torch.zeros_like(good[2])
    bad = c.pages.clone()
    bad[int(c.base[7])] = 10_000
    wrong = ro.ro_cache(c.k.cuda(), c.v.cuda(), i64(c.base), bad.cuda())
    ok(ctx, ro.ro_cache_attend(ctx, wrong, i64(range(401)), 1, i32(lens), 40, good[1], 0.1, 0, 0, out))
    assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
    rest = [s for s in range(400) if s != 7]
    assert torch.equal(out[rest], good[2][rest])
    ok(ctx, ro.ro_cache_attend(ctx, cache, i64(range(401)), 1, i32([500] + lens[1:]), 40, good[1], 0.1, 0, 0, out))
    assert ro.ro_ctx_sync(ctx) == ro.RO_E_CAPACITY


@pytest.mark.parametrize("heads,kv", [(4, 2), (8, 1)])
@pytest.mark.parametrize("news", [[40, 300], [1, 5]])
def test_attend_rows_that_see_nothing(ctx, heads, kv, news):
    """A chunk longer than what the cache holds: its first tokens lie before slot 0."""
    lens = [7, 260] if news[0] > 1 else [0, 2]
    c = ref.Cache([max(L, 1) for L in lens], kv, 64, 16, BF16, 2)
    c.lens = lens
    out, lse = check_attend(ctx, c, news, heads)
    assert bool((out[0] == 0).all()) and bool(torch.isinf(lse[0]).all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
@pytest.mark.parametrize("news", [[1, 1], [90, 40]])
def test_attend_scales(ctx, scale, news):
    check_attend(ctx, ref.Cache([500, 90], 2, 64, 32, BF16, 8), news, 4, scale=scale)


def test_attend_splits_and_joins(ctx):
    """A long cache and few rows: keys split over the GPU, joined in order; equal calls give equal bits, and the
    guess of the length changes the split alone."""
    c = ref.Cache([9000, 3], 2, 64, 64, BF16, 4)
    out, lse = check_attend(ctx, c, [2, 3], 4)
    for max_len in (0, 100, 9000, 1 << 30):
        o2, l2 = check_attend(ctx, c, [2, 3], 4, max_len=max_len)
    o2, l2 = check_attend(ctx, c, [2, 3], 4)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_attend_kernels_share_a_context(ctx):
    """Calls that split and join in different ways, one after another on one context's workspaces."""
    few = ref.Cache([3000, 2500, 900], 2, 64, 64, BF16, 41)
    some = ref.Cache([4000, 60], 2, 64, 64, BF16, 42)
    odd = ref.Cache([2500, 300], 2, 64, 7, BF16, 43)
    want = {}
    for _ in range(2):
        for name, c, news in (("few", few, [1, 2, 1]), ("some", some, [40, 60]), ("odd", odd, [30, 9]), ("some", some, [40, 60]),
                              ("few", few, [1, 2, 1])):
            got = check_attend(ctx, c, news, 4)
            for a, b in zip(got, want.setdefault(name, got)):
                assert torch.equal(a, b)


@pytest.mark.parametrize("news", [[1, 1], [50, 90]])
@pytest.mark.parametrize("window,sinks", [(2 ** 32 - 1, 0), (2 ** 31, 5), (2 ** 31 - 1, 0), (3, 2 ** 32 - 1), (70, 2 ** 31)])
def test_attend_and_weigh_windows_past_every_slot(ctx, news, window, sinks):
    """Windows and sinks wider than any cache: the same as none (and as everything)."""
    lens = [400, 90]
    c = ref.Cache(lens, 2, 64, 16, BF16, 44)
    q, dq, out, lse = run_attend(ctx, c, news, 4, 0.125, window, sinks)
    _, _, want, want_lse = run_attend(ctx, c, news, 4, 0.125, 0, 0)
    cache, _, _ = on_gpu(c)
    scores = [torch.zeros(2, 2, 400, device="cuda") for _ in range(2)]
    for score, w, k in zip(scores, (window, 0), (sinks, 0)):
        ok(ctx, ro.ro_cache_weigh(ctx, cache, i64(starts(news)), max(news), i32(lens), dq, 0.125, w, k, lse, 1.0, None, score))
    sync_ok(ctx)
    if sinks < 2 ** 31:   # the same slots in the same order: the same bits
        assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(*scores)
    else:
        t = starts(news)
        for s in range(2):
            w_out, w_lse, tol, lse_tol = ref.attend(c, s, q[t[s]:t[s + 1]], 0.125, 0, 0)
            within(out[t[s]:t[s + 1]], w_out, tol)
            within(lse[t[s]:t[s + 1]], w_lse, lse_tol)
            w, wtol = ref.weigh(c, s, q[t[s]:t[s + 1]], 0.125, 0, 0, lse[t[s]:t[s + 1]].double().cpu(), 1.0,
                                torch.zeros(2, lens[s]))
            within(scores[0][s, :, :lens[s]], w, wtol + 1e-30)


@pytest.mark.parametrize("page", [16, 20, 256])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_long_runs(ctx, dim, page):
    """Enough sequences that a CTA goes round its ring of stages many times."""
    g = np.random.default_rng(page)
    lens = [int(x) for x in g.integers(3000, 6000, 44)]
    check_attend(ctx, ref.Cache(lens, 7, dim, page, BF16, page), [1] * 44, 7)


@pytest.mark.parametrize("heads,kv", [(4, 4), (14, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 5)])
def test_attend_many_row_tiles(ctx, heads, kv, window, sinks):
    """Chunks of more row tiles than the GPU has places for, of uneven sequences."""
    lens, news = [900, 2100, 300, 1500], [900, 600, 1, 1100]
    c = ref.Cache(lens, kv, 64, 32, F16, 31)
    scale = 0.125
    q, _, out, lse = run_attend(ctx, c, news, heads, scale, window, sinks)
    t = starts(news)
    for s in range(4):
        for i in sorted({0, news[s] // 2, news[s] - 1}):   # some rows of each chunk
            c.lens = list(lens)
            c.lens[s] = lens[s] - news[s] + i + 1          # the row is the last of its cache
            w_out, w_lse, tol, lse_tol = ref.attend(c, s, q[t[s] + i:t[s] + i + 1], scale, window, sinks)
            within(out[t[s] + i:t[s] + i + 1], w_out, tol)
            within(lse[t[s] + i:t[s] + i + 1], w_lse, lse_tol)


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), 6e4])
@pytest.mark.parametrize("news", [[1, 1], [64, 30]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_attend_never_uses_unseen_slots(ctx, junk, news, window, sinks):
    """Stale slots past the length, unused pages, and slots between the sinks and every token's window."""
    lens = [201, 67]
    c = ref.Cache(lens, 1, 64, 16, F16, 6, junk=junk)
    clean = ref.Cache(lens, 1, 64, 16, F16, 6, junk=0.0)
    if window:
        for s, L in enumerate(lens):
            for j in range(sinks, L - news[s] - window + 1):
                at, slot = int(c.pages[c.base[s] + j // 16]), j % 16
                c.k[at, :, slot] = junk
                c.v[at, :, slot] = junk
    got = run_attend(ctx, c, news, 4, 0.125, window, sinks)
    want = run_attend(ctx, clean, news, 4, 0.125, window, sinks)
    assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])


def test_attend_offsets_past_32_bits(ctx):
    """Pools of more than 2^32 elements."""
    stride = 1 << 31
    c = ref.Cache([150], 2, 64, 64, BF16, 9, spare=0)
    pools = []
    for pool in (c.k, c.v):
        flat = torch.empty(2 * stride + 2 * 64 * 64, dtype=BF16, device="cuda")
        big = flat.as_strided((3, 2, 64, 64), (stride, 64 * 64, 64, 1))
        big.copy_(pool.cuda())
        pools.append(big)
    cache = ro.ro_cache(pools[0], pools[1], i64(c.base), c.pages.cuda())
    for news in ([1], [100]):
        check_attend(ctx, c, news, 4, gpu=(cache, None, None))


def test_attend_bad_pages_and_ranges_are_recorded(ctx):
    c = ref.Cache([100, 40], 1, 64, 16, BF16, 3, junk=0.0)
    want = run_attend(ctx, c, [1, 1], 2, 0.1, 0, 0)[2]
    for news in ([1, 1], [40, 40]):
        c.pages[1] = 10_000
        cache = on_gpu(c)
        T = sum(news)
        q = torch.zeros(T, 2, 64, dtype=BF16, device="cuda")
        out = torch.zeros_like(q)
        ok(ctx, ro.ro_cache_attend(ctx, cache[0], i64(starts(news)), max(news), i32(c.lens), 100, q, 0.1, 0, 0, out))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
        c.pages[1] = int(c.free[0])
        cache = on_gpu(c)
        ok(ctx, ro.ro_cache_attend(ctx, cache[0], i64(starts(news)), max(news), i32([500, 40]), 100, q, 0.1, 0, 0, out))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_CAPACITY
        ok(ctx, ro.ro_cache_attend(ctx, cache[0], i64([0, T + 5, T]), max(news), i32(c.lens), 100, q, 0.1, 0, 0, out))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
    # a sequence with more than max_new tokens is left out, the others are not
    q = torch.randn(3, 2, 64, device="cuda").to(BF16)
    out = torch.full_like(q, 5)
    ok(ctx, ro.ro_cache_attend(ctx, cache[0], i64([0, 2, 3]), 1, i32(c.lens), 100, q, 0.1, 0, 0, out))
    assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
    assert bool((out[:2] == 5).all()) and not bool((out[2] == 5).any()) and want is not None
    sync_ok(ctx)


def test_attend_on_another_stream_and_in_a_graph(ctx):
    c = ref.Cache([3000, 400], 2, 64, 64, BF16, 10)
    cache, _, _ = on_gpu(c)
    side = torch.cuda.Stream()
    c2 = ro.ro_ctx_create(0, side, 1)
    for news in ([1, 1], [150, 90]):
        q, dq, out, lse = run_attend(ctx, c, news, 4, 0.125, 0, 0)
        base, lens = i64(starts(news)), i32(c.lens)
        o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
        side.wait_stream(torch.cuda.current_stream())

        def call():
            ok(c2, ro.ro_cache_attend(c2, cache, base, max(news), lens, 3000, dq, 0.125, 0, 0, o2, l2))

        call()
        sync_ok(c2)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for _ in range(2):
            o2.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, o2) and torch.equal(lse, l2)
    ro.ro_ctx_destroy(c2)


# ---------------------------------------------------------------------------- weigh
@pytest.mark.parametrize("dtype,dim,heads,kv,page", [(BF16, 128, 4, 2, 64), (F16, 64, 3, 3, 16), (BF16, 80, 6, 1, 20),
                                                     (F16, 40, 9, 3, 5)])
@pytest.mark.parametrize("news,window,sinks", [([1, 1, 0, 1], 0, 0), ([40, 1, 0, 131], 0, 0), ([40, 1, 0, 131], 16, 5),
                                               ([1, 1, 0, 1], 9, 0), ([200, 129, 40, 1], 0, 0)])
def test_weigh(ctx, dtype, dim, heads, kv, page, news, window, sinks):
    lens = [200, 129, 40, 140]
    c = ref.Cache(lens, kv, dim, page, dtype, 12)
    scale = 1 / math.sqrt(dim)
    q, dq, _, lse = run_attend(ctx, c, news, heads, scale, window, sinks)
    cache, _, _ = on_gpu(c)
    cap = 211
    past = torch.rand(4, kv, cap).cuda()
    score = torch.full((4, kv, cap), -5.0, device="cuda")
    base = i64(starts(news))
    ok(ctx, ro.ro_cache_weigh(ctx, cache, base, max(news), i32(lens), dq, scale, window, sinks, lse, 0.75, past, score))
    in_place = past.clone()
    ok(ctx, ro.ro_cache_weigh(ctx, cache, base, max(news), i32(lens), dq, scale, window, sinks, lse, 0.75, in_place,
                              in_place))
    fresh = torch.full((4, kv, cap), -5.0, device="cuda")
    ok(ctx, ro.ro_cache_weigh(ctx, cache, base, 0, i32(lens), dq, scale, window, sinks, lse, 1.0, None, fresh))
    sync_ok(ctx)
    t = starts(news)
    for s, L in enumerate(lens):
        for got, pst in ((score, past), (fresh, past * 0)):
            want, tol = ref.weigh(c, s, q[t[s]:t[s + 1]], scale, window, sinks, lse[t[s]:t[s + 1]].double().cpu(),
                                  0.75, pst[s].cpu())
            within(got[s, :, :L], want, tol + 1e-30)
            assert bool((got[s, :, L:] == -5).all())
        assert torch.equal(in_place[s, :, :L], score[s, :, :L])
        assert torch.equal(in_place[s, :, L:], past[s, :, L:])


@pytest.mark.parametrize("page", [64, 20])
@pytest.mark.parametrize("heads,kv,news,window,sinks", [(4, 4, 1, 0, 0), (16, 2, 2, 1000, 9), (6, 2, 300, 0, 0),
                                                        (14, 2, 130, 900, 0)])
def test_weigh_long_runs(ctx, page, heads, kv, news, window, sinks):
    """Many stages and row tiles a CTA; the weights of a row add up to one."""
    g = np.random.default_rng(heads)
    lens = [int(x) for x in g.integers(2000, 5000, 70 if news < 3 else 3)]
    c = ref.Cache(lens, kv, 128, page, BF16, page)
    n = [news] * len(lens)
    q, dq, _, lse = run_attend(ctx, c, n, heads, 0.088, window, sinks)
    cache, _, _ = on_gpu(c)
    score = torch.zeros(len(lens), kv, max(lens), device="cuda")
    ok(ctx, ro.ro_cache_weigh(ctx, cache, i64(starts(n)), news, i32(lens), dq, 0.088, window, sinks, lse, 1.0, None, score))
    sync_ok(ctx)
    # each of news * heads / kv rows gives 1 in all; a weight errs by its exponent's 32 bits (|x| < 64: 2^-18) and the lse's
    total = score.double().sum(2).cpu()
    want = torch.full_like(total, news * heads / kv)
    assert bool(((total - want).abs() <= want * 2.0 ** -16).all())
    for s in (0, len(lens) - 1):
        if news > 2:
            continue
        w, tol = ref.weigh(c, s, q[s * news:(s + 1) * news], 0.088, window, sinks,
                           lse[s * news:(s + 1) * news].double().cpu(), 1.0, torch.zeros(kv, max(lens)))
        within(score[s, :, :lens[s]], w, tol + 1e-30)


def test_weigh_rows_that_see_nothing_and_short_scores(ctx):
    c = ref.Cache([7], 1, 64, 16, BF16, 13)
    q, dq, _, lse = run_attend(ctx, c, [30], 2, 0.125, 0, 0)
    cache, _, _ = on_gpu(c)
    score = torch.zeros(1, 1, 7, device="cuda")
    ok(ctx, ro.ro_cache_weigh(ctx, cache, i64([0, 30]), 30, i32([7]), dq, 0.125, 0, 0, lse, 1.0, None, score))
    sync_ok(ctx)
    want, tol = ref.weigh(c, 0, q, 0.125, 0, 0, lse.double().cpu(), 1.0, torch.zeros(1, 7))
    within(score[0], want, tol + 1e-30)
    short = torch.zeros(1, 1, 5, device="cuda")
    ok(ctx, ro.ro_cache_weigh(ctx, cache, i64([0, 30]), 30, i32([7]), dq, 0.125, 0, 0, lse, 1.0, None, short))
    assert ro.ro_ctx_sync(ctx) == ro.RO_E_CAPACITY


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 5), (70, 130), (64, 64), (500, 1)])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 20), (40, 5)])
@pytest.mark.parametrize("cap", [3000, 3001])
def test_weigh_few_rows_behind_a_window(ctx, window, sinks, dim, page, cap):
    """What no row sees only has its past decayed, wherever it starts and ends; rows of scores aligned and not."""
    lens, news = [1000, 513, 64, 3000, 0, 700, 65], [1, 3, 1, 2, 0, 0, 1]
    c = ref.Cache(lens, 2, dim, page, F16, 41)
    scale = 1 / math.sqrt(dim)
    q, dq, _, lse = run_attend(ctx, c, news, 4, scale, window, sinks)
    cache, _, _ = on_gpu(c)
    past = torch.rand(7, 2, cap).cuda()
    score, in_place = torch.full_like(past, -5.0), past.clone()
    for before, out in ((past, score), (in_place, in_place)):
        ok(ctx, ro.ro_cache_weigh(ctx, cache, i64(starts(news)), 3, i32(lens), dq, scale, window, sinks, lse, 0.75, before,
                                  out))
    sync_ok(ctx)
    t = starts(news)
    for s, L in enumerate(lens):
        want, tol = ref.weigh(c, s, q[t[s]:t[s + 1]], scale, window, sinks, lse[t[s]:t[s + 1]].double().cpu(), 0.75,
                              past[s].cpu())
        within(score[s, :, :L], want, tol + 1e-30)
        assert bool((score[s, :, L:] == -5).all())
        assert torch.equal(in_place[s, :, :L], score[s, :, :L]) and torch.equal(in_place[s, :, L:], past[s, :, L:])


@pytest.mark.parametrize("window,sinks", [(0, 0), (48, 3)])
@pytest.mark.parametrize("dim,heads,kv", [(64, 6, 2), (128, 4, 4)])
def test_weigh_many_sequences(ctx, window, sinks, dim, heads, kv):
    """Chunks of 75 sequences, some empty, some without new tokens: CTAs take many of them in turn."""
    g = np.random.default_rng(dim + window)
    lens = [int(x) for x in g.integers(0, 900, 75)]
    news = [min(L, int(x)) for L, x in zip(lens, g.integers(0, 60, 75))]
    for s in (0, 31, 32, 74):
        lens[s] = news[s] = 0
    for s in (5, 40, 73):
        news[s] = 0
    c = ref.Cache(lens, kv, dim, 16, BF16, 29)
    scale = 1 / math.sqrt(dim)
    q, dq, _, lse = run_attend(ctx, c, news, heads, scale, window, sinks)
    cache, _, _ = on_gpu(c)
    cap = max(lens)
    past = torch.rand(len(lens), kv, cap).cuda()
    scores = [torch.full((len(lens), kv, cap), -5.0, device="cuda") for _ in range(3)]
    for score in scores:
        ok(ctx, ro.ro_cache_weigh(ctx, cache, i64(starts(news)), 60, i32(lens), dq, scale, window, sinks, lse, 0.5, past,
                                  score))
    sync_ok(ctx)
    assert torch.equal(scores[0], scores[1]) and torch.equal(scores[0], scores[2])   # whoever took what
    t = starts(news)
    for s, L in enumerate(lens):
        assert bool((scores[0][s, :, L:] == -5).all())
        if s % 6 == 0 or news[s] == 0:
            want, tol = ref.weigh(c, s, q[t[s]:t[s + 1]], scale, window, sinks, lse[t[s]:t[s + 1]].double().cpu(), 0.5,
                                  past[s].cpu())
            within(scores[0][s, :, :L], want, tol + 1e-30)


def test_weigh_bad_ranges_are_recorded_and_the_next_call_is_whole(ctx):
    lens, news = [300] * 40, [20] * 40
    c = ref.Cache(lens, 1, 64, 16, BF16, 31)
    q, dq, _, lse = run_attend(ctx, c, news, 2, 0.125, 0, 0)
    cache, _, _ = on_gpu(c)
    base = starts(news)
    good = torch.zeros(40, 1, 300, device="cuda")
    ok(ctx, ro.ro_cache_weigh(ctx, cache, i64(base), 20, i32(lens), dq, 0.125, 0, 0, lse, 1.0, None, good))
    sync_ok(ctx)
    bad = base.copy()
    bad[38] = 10_000                      # the ranges of sequences 37 and 38
    score = torch.full_like(good, -5.0)
    ok(ctx, ro.ro_cache_weigh(ctx, cache, i64(bad), 20, i32(lens), dq, 0.125, 0, 0, lse, 1.0, None, score))
    assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
    assert bool((score[37:39] == -5).all())
    assert torch.equal(score[:37], good[:37]) and torch.equal(score[39:], good[39:])
    other = ro.ro_ctx_create(0, torch.cuda.current_stream(), 1)
    try:
        again = torch.zeros_like(good)
        ok(other, ro.ro_cache_weigh(other, cache, i64(base), 20, i32(lens), dq, 0.125, 0, 0, lse, 1.0, None, again))
        sync_ok(other)
        assert torch.equal(again, good)
    finally:
        ro.ro_ctx_destroy(other)


# ---------------------------------------------------------------------------- evict
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (64, 4, 16), (100, 0, 0), (100, 50, 50),
                                                 (999, 3, 7), (1000, 0, 0), (4000, 4, 100)])
@pytest.mark.parametrize("kind", ["tail", "ties", "nan", "signed"])
def test_evict(ctx, budget, sinks, recent, kind):
    lens, kv, dim, page = [1000, 64, 0, 3000, 65], 2, 72, 16
    c = ref.Cache(lens, kv, dim, page, BF16, 21, junk=1.0)
    g = torch.Generator().manual_seed(budget)
    cap = 3001
    x = torch.randn(len(lens), kv, cap, generator=g)
    score = {"tail": (3 * x).exp(), "ties": x.abs().floor(), "signed": torch.where(x.abs() < 0.1, x * 0, x),
             "nan": torch.where(x > 1.5, torch.full_like(x, math.nan), torch.where(x < -2, x / 0, x))}[kind]
    kept = [min(L, budget) for L in lens]
    need = [-(-n // page) for n in kept]
    src, total = c.k.shape[0], c.k.shape[0] + sum(need)
    k, v = (torch.cat([p, torch.zeros(sum(need), kv, page, dim, dtype=BF16)]).cuda() for p in (c.k, c.v))
    dst_base = starts(need)
    dst = src + torch.randperm(sum(need), generator=g).int()
    cache = ro.ro_cache(k, v, i64(c.base), c.pages.cuda())
    keep = torch.full((len(lens), kv, budget), -1, dtype=torch.int32, device="cuda")
    len_out = torch.full((len(lens),), 77, dtype=torch.int32, device="cuda")
    out = torch.full_like(score, -7.0).cuda()
    before_k, before_v = k.cpu(), v.cpu()
    ok(ctx, ro.ro_cache_evict(ctx, cache, i32(lens), score.cuda(), budget, sinks, recent, i64(dst_base), dst.cuda(), keep,
                              len_out, out))
    sync_ok(ctx)
    assert len_out.tolist() == kept
    want_k, want_v = before_k.clone(), before_v.clone()
    for s, L in enumerate(lens):
        for h in range(kv):
            idx = ref.evict(L, score[s, h].numpy(), budget, sinks, recent)
            n = kept[s]
            assert np.array_equal(keep[s, h, :n].cpu().numpy(), idx) and bool((keep[s, h, n:] == -1).all())
            got = out[s, h].cpu()
            assert np.array_equal(got[:n].numpy(), score[s, h].numpy()[idx], equal_nan=True) and bool((got[n:] == -7).all())
            j, d = torch.as_tensor(idx), torch.arange(n)
            at = dst[dst_base[s] + d // page].long()
            page_of = c.pages[c.base[s] + j // page].long()
            want_k[at, h, d % page] = before_k[page_of, h, j % page]
            want_v[at, h, d % page] = before_v[page_of, h, j % page]
    assert total == k.shape[0] and torch.equal(k.cpu(), want_k) and torch.equal(v.cpu(), want_v)


@pytest.mark.parametrize("lens,kv,budget,sinks,recent", [([40_000, 9_000], 2, 700, 4, 100), ([200_000], 1, 20_000, 0, 0),
                                                         ([30_000, 0, 12_000, 8_200], 1, 8_192, 16, 8_000),
                                                         ([33_333], 3, 33_332, 1, 5), ([20_000] * 3, 2, 50, 20, 30)])
@pytest.mark.parametrize("kind", ["tail", "ties", "same"])
def test_evict_long_sequences(ctx, lens, kv, budget, sinks, recent, kind):
    """Sequences that several CTAs share: kept slots and scores (rows of 8 dimensions stand for the rest)."""
    g = torch.Generator().manual_seed(len(lens))
    page, cap = 128, max(lens) + 3
    x = torch.randn(len(lens), kv, cap, generator=g)
    score = {"tail": (3 * x).exp(), "ties": (x.abs() * 4).floor(), "same": x * 0 + 1.5}[kind]
    held = [-(-L // page) for L in lens]
    need = [-(-min(L, budget) // page) for L in lens]
    k = torch.arange((sum(held) + sum(need)) * kv * page * 8, device="cuda").view(-1, kv, page, 8).to(BF16)
    v = -k
    cache = ro.ro_cache(k, v, i64(starts(held)), i32(np.arange(sum(held))))
    before = k.clone()
    keep = torch.full((len(lens), kv, budget), -1, dtype=torch.int32, device="cuda")
    n_out = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    out = torch.full_like(score, -7.0).cuda()
    ok(ctx, ro.ro_cache_evict(ctx, cache, i32(lens), score.cuda(), budget, sinks, recent, i64(starts(need)),
                              i32(sum(held) + np.arange(sum(need))), keep, n_out, out))
    sync_ok(ctx)
    for s, L in enumerate(lens):
        for h in range(kv):
            idx = ref.evict(L, score[s, h].numpy(), budget, sinks, recent)
            n = len(idx)
            assert np.array_equal(keep[s, h, :n].cpu().numpy(), idx)
            assert np.array_equal(out[s, h, :n].cpu().numpy(), score[s, h].numpy()[idx])
            j, d = torch.as_tensor(idx).cuda(), torch.arange(n, device="cuda")
            at = sum(held) + starts(need)[s] + d // page
            assert torch.equal(k[at, h, d % page], before[starts(held)[s] + j // page, h, j % page])
            assert torch.equal(v[at, h, d % page], -before[starts(held)[s] + j // page, h, j % page])


def test_evict_records_what_does_not_fit(ctx):
    c = ref.Cache([40], 1, 8, 4, BF16, 22, spare=4, junk=0.0)
    score = torch.rand(1, 1, 40).cuda()

    def call(dst_base, dst, lens, cap=40):
        cache, k, v = on_gpu(c)
        keep = torch.zeros(1, 1, 10, dtype=torch.int32, device="cuda")
        n = torch.zeros(1, dtype=torch.int32, device="cuda")
        ok(ctx, ro.ro_cache_evict(ctx, cache, i32(lens), score[:, :, :cap].contiguous(), 10, 0, 0, i64(dst_base),
                                  i32(dst), keep, n))
        return ro.ro_ctx_sync(ctx), k

    free = c.free.tolist()
    st, _ = call([0, 3], free[:3], [40])
    assert st == ro.RO_OK
    st, k = call([0, 2], free[:2], [40])
    assert st == ro.RO_E_CAPACITY and bool((k[free[2]] == 0).all())
    st, k = call([0, 3], free[:2] + [999], [40])
    assert st == ro.RO_E_INVAL and bool((k[free[2]] == 0).all())
    assert call([0, 3], free[:3], [44])[0] == ro.RO_E_CAPACITY
    assert call([0, 3], free[:3], [40], cap=30)[0] == ro.RO_E_CAPACITY
    sync_ok(ctx)


# ---------------------------------------------------------------------------- refusals
def test_refusals(ctx):
    k = torch.zeros(4, 2, 16, 64, dtype=BF16, device="cuda")
    base, pages, lens = i64([0, 4]), i32([0, 1, 2, 3]), i32([10])
    cache = ro.ro_cache(k, k.clone(), base, pages)
    q = torch.zeros(3, 4, 64, dtype=BF16, device="cuda")
    lse = torch.zeros(3, 4, device="cuda")
    tok = i64([0, 3])
    pos = i32(np.zeros((3, 1)))

    def attend(cache=cache, q=q, scale=1.0, out=None):
        out = torch.zeros_like(q) if out is None else out
        return ro.ro_cache_attend(ctx, cache, tok, 3, lens, 10, q, scale, 0, 0, out, None)

    ok(ctx, attend())
    assert attend(q=torch.zeros(3, 3, 64, dtype=BF16, device="cuda")) == ro.RO_E_INVAL   # 3 heads over 2
    assert "multiple" in ro.ro_last_error(ctx)
    assert attend(scale=math.inf) == ro.RO_E_INVAL
    off = torch.zeros(3 * 4 * 64 + 8, dtype=BF16, device="cuda")[1:1 + 3 * 4 * 64].view(3, 4, 64)
    assert attend(q=off) == ro.RO_E_INVAL
    assert attend(out=off) == ro.RO_E_INVAL
    wide = torch.zeros(4, 2, 16, 136, dtype=BF16, device="cuda")
    assert attend(cache=ro.ro_cache(wide, wide.clone(), base, pages), q=torch.zeros(3, 4, 136, dtype=BF16, device="cuda")) \
        == ro.RO_E_INVAL
    odd = torch.zeros(4, 2, 16, 68, dtype=BF16, device="cuda")
    assert attend(cache=ro.ro_cache(odd[..., :64], odd.clone()[..., :64], base, pages)) == ro.RO_E_INVAL
    for rope in (ro.ro_rope([33]), ro.ro_rope([0, 0]), ro.ro_rope([8], base=0.5), ro.ro_rope([8], base=math.nan)):
        p = i32(np.zeros((3, rope.n_axes)))
        assert ro.ro_rotary(ctx, q, q.clone(), p, rope) == ro.RO_E_INVAL
        assert ro.ro_cache_append(ctx, cache, tok, i32([0, 0, 0]), lens, p, rope, q, q.clone(), q[:, :2], q[:, 2:]) \
            == ro.RO_E_INVAL
    assert ro.ro_rotary(ctx, torch.zeros(3, 2, 258, device="cuda"), torch.zeros(3, 2, 258, device="cuda"), pos,
                        ro.ro_rope([8])) == ro.RO_E_INVAL
    score = torch.zeros(1, 2, 64, device="cuda")
    assert ro.ro_cache_weigh(ctx, cache, tok, 3, lens, q, 1.0, 0, 0, lse, math.nan, None, score) == ro.RO_E_INVAL
    keep = torch.zeros(1, 2, 8, dtype=torch.int32, device="cuda")

    def evict(sinks=0, recent=0, out=None):
        return ro.ro_cache_evict(ctx, cache, lens, score, 8, sinks, recent, i64([0, 1]), i32([3]), keep, lens.clone(), out)

    assert evict(sinks=5, recent=4) == ro.RO_E_INVAL
    assert evict(out=score) == ro.RO_E_INVAL
    with pytest.raises(ValueError):
        attend(q=q.half())
    with pytest.raises(ValueError):
        ro.ro_cache(k, k[:2], base, pages)
    with pytest.raises(ValueError):
        ro.ro_cache_attend(ctx, cache, tok.int(), 3, lens, 10, q, 1.0, 0, 0, q.clone())
    ok(ctx, ro.ro_cache_attend(ctx, cache, i64([0, 0]), 0, lens, 10, q[:0], 1.0, 0, 0, q[:0].clone()))   # no tokens
    sync_ok(ctx)
