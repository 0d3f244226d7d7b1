"""Sampling on the GPU against its definition in 64 bits: tokens and counts are
equal, at every combination of settings, ties, masked and infinite logits, odd
vocabularies, strides and alignments."""
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

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NONE = -1   # RO_NO_TOKEN as a signed integer


@pytest.fixture
def ctx():
    c = ro.ro_ctx_create(0, torch.cuda.current_stream(), 1)
    yield c
    ro.ro_ctx_destroy(c)


def ok(ctx, status):
    assert status == ro.RO_OK, ro.ro_last_error(ctx)


def draw(x, t, k, p, m, u):
    """One row from its definition: token, how many stay, ln of its share."""
    x = np.where(np.isnan(x), -np.inf, x)
    V = x.size
    order = np.lexsort((np.arange(V), -x))
    order = order[: int((x > -np.inf).sum())]
    if order.size == 0:
        return NONE, 0, -math.inf
    if t == 0:
        return int(order[0]), 1, 0.0
    with np.errstate(invalid="ignore"):
        w = np.exp(np.where(x[order] == x[order[0]], 0.0, (x[order] - x[order[0]]) / t))
    first = order.size if k == 0 else min(k, order.size)
    count = first
    if p < 1:
        ahead = np.concatenate([[0.0], np.cumsum(w[:first])[:-1]])
        count = max(1, int((ahead < p * math.fsum(w[:first])).sum()))
    count = min(count, int((w >= m).sum()))
    order, w = order[:count], w[:count]
    place = np.argsort(order)
    runs = np.cumsum(w[place])
    hit = place[int(np.searchsorted(runs, u * runs[-1], side="right"))]
    return int(order[hit]), count, math.log(w[hit] / runs[-1])


def check(ctx, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, device=None):
    n, V = logits.shape
    dev = logits.cuda() if device is None else device
    f = lambda v, d: None if v is None else torch.tensor(np.broadcast_to(np.asarray(v), (n,)).copy(), dtype=d).cuda()   # noqa: E731
    how = ro.ro_sampling(f(temperature, F32), f(top_k, torch.int32), f(top_p, F32), f(min_p, F32))
    token, kept = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    logp = torch.full((n,), 7.0, device="cuda")
    du = torch.as_tensor(u, dtype=F32).cuda()
    ok(ctx, ro.ro_sample(ctx, dev, how, du, token, logp, kept))
    ok(ctx, ro.ro_ctx_sync(ctx))
    x, us = logits.double().numpy(), du.double().cpu().numpy()
    g = lambda v, r: None if v is None else v[r].item()   # noqa: E731
    for r in range(n):
        t, k, p, m = (g(z, r) for z in how._tensors)
        want = draw(x[r], 1.0 if t is None else t, 0 if k is None else k & 0xFFFFFFFF, 1.0 if p is None else p,
                    0.0 if m is None else m, us[r])
        assert (token[r].item(), kept[r].item()) == want[:2], (r, want, t, k, p, m)
        # the difference of logits in 64 bits, one rounding to 32: half a step, and the weights' 2^-39
        assert logp[r].item() == want[2] or abs(logp[r].item() - want[2]) <= 2.0 ** -23 * abs(want[2]) + 2.0 ** -36
    return token, logp, kept


def rows(n, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, V, generator=g) * spread
    hot = torch.randint(0, V, (n, 8), generator=g)
    x.scatter_add_(1, hot, torch.randn(n, 8, generator=g) * 3 + 3)
    return x.to(dtype), torch.rand(n, generator=g)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 4099, 32_000, 131_072, 200_003])
@pytest.mark.parametrize("settings", [(), ("t",), ("k",), ("p",), ("m",), ("t", "k", "p"), ("t", "p", "m"), ("t", "k", "p", "m")])
def test_draws(ctx, dtype, V, settings):
    n = 24 if V < 50_000 else 6
    x, u = rows(n, V, dtype, V + len(settings))
    g = np.random.default_rng(V)
    pick = {"t": ("temperature", g.uniform(0.3, 2.0, n)), "k": ("top_k", g.integers(0, min(2 * V, 300) + 1, n)),
            "p": ("top_p", g.uniform(0.05, 0.999, n)), "m": ("min_p", g.uniform(0.0, 0.3, n))}
    check(ctx, x, u, **dict(pick[s] for s in settings))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_flat_rows_keep_many(ctx, dtype):
    """Nuclei and top-k of tens of thousands of tokens, many of them equal."""
    x, u = rows(6, 60_000, dtype, 3, spread=0.2)
    check(ctx, x, u, top_p=[0.5, 0.9, 0.99, 0.999999, 0.3, 0.1], temperature=[1, 3, 0.5, 1, 2, 1])
    check(ctx, x, u, top_k=[50_000, 30_000, 5000, 59_999, 60_000, 2049], top_p=[0.5, 0.9, 1, 0.8, 0.7, 0.9])
    check(ctx, x, u, min_p=[0.01, 0.5, 0.9, 1.0, 0.2, 0.7], top_p=[0.9, 0.8, 0.99, 0.5, 1.0, 0.0])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_ties_go_to_the_lowest_index(ctx, dtype):
    n, V = 8, 3000
    x = torch.zeros(n, V, dtype=dtype)
    u = torch.linspace(0, 0.999, n)
    check(ctx, x, u, top_k=[1, 2, 10, 999, 3000, 0, 2500, 7])
    check(ctx, x, u, top_p=[0.5, 0.25, 0.9, 0.1, 1.0, 0.0, 0.75, 0.999])
    check(ctx, x, u, top_k=1000, top_p=0.5, min_p=1.0)
    x[:, 1::2] = -0.0                      # the same number
    check(ctx, x, u, top_k=[1, 2, 10, 999, 3000, 0, 2500, 7], top_p=0.5)
    x[:, ::3] = 1.0                        # the border inside a run of equal ones
    x[:, 5::7] = -2.0
    check(ctx, x, u, top_k=[1500, 1001, 1003, 2600, 2999, 1000, 999, 1], top_p=[1, 0.9, 0.99, 0.7, 0.95, 0.6, 0.5, 0.4])
    check(ctx, x, u, temperature=0.0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V", [5, 5000, 140_001])
def test_masked_and_infinite_logits(ctx, dtype, V):
    x, u = rows(10, V, dtype, 9)
    low = torch.finfo(dtype).min
    x[0] = -math.inf                       # nothing to draw
    x[1] = math.nan
    x[2] = -math.inf
    x[2, V - 1] = low                      # one token, whatever its logit
    x[3, ::2] = -math.inf
    x[4, ::3] = math.nan
    x[5, 2], x[5, V - 1] = math.inf, math.inf
    x[6] = low                             # all alike, at the type's lowest value
    x[7, 1:] = low
    x[8, ::2] = low
    x[9, 0] = torch.finfo(dtype).max
    for kw in (dict(), dict(top_k=3), dict(top_p=0.7), dict(min_p=0.05), dict(top_k=40, top_p=0.9, min_p=0.01, temperature=1.7),
               dict(temperature=0.0), dict(top_p=0.0)):
        check(ctx, x, u, **kw)


@pytest.mark.parametrize("temperature", [1e-45, 1e-30, 1e-3, 0.05, 50.0, 1e6, 3e38])
def test_temperatures(ctx, temperature):
    x, u = rows(6, 9000, F32, 2)
    check(ctx, x, u, temperature=temperature)
    check(ctx, x, u, temperature=temperature, top_k=100, top_p=0.8)


def test_random_numbers_at_the_ends(ctx):
    x, _ = rows(6, 5000, BF16, 4)
    x[:, 0] = -math.inf
    u = torch.tensor([0.0, 1e-45, 2.0 ** -24, 0.5, 1 - 2.0 ** -24, 1 - 2.0 ** -23])
    for kw in (dict(), dict(top_k=50), dict(top_p=0.9), dict(top_p=1e-45), dict(top_p=1 - 2.0 ** -24), dict(min_p=1e-40)):
        check(ctx, x, u, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (2, 1), (7, 9)])
def test_strides_and_alignment(ctx, dtype, offset, pad):
    """Rows at any alignment, junk around them."""
    n, V = 9, 2051
    x, u = rows(n, V, dtype, 6)
    buf = torch.full((offset + n * (V + pad) + 16,), math.inf, dtype=dtype, device="cuda")
    view = buf[offset:offset + n * (V + pad)].view(n, V + pad)[:, :V]
    view.copy_(x)
    check(ctx, x, u, device=view, top_p=0.9, top_k=[0, 1, 5, 70, 2051, 9999, 0, 33, 2])
    one = x[:1].cuda().expand(n, V)        # many draws of one row
    check(ctx, x[:1].expand(n, V), u, device=one, temperature=1.3)


def test_every_row_count_draws_alike(ctx):
    """How a row is split over the GPU depends on the number of rows; what it draws does not."""
    x, u = rows(700, 10_007, BF16, 8)
    kw = dict(temperature=0.9, top_k=torch.arange(700) % 90, top_p=0.95)
    dev = x.cuda()
    base = None
    for n in (700, 300, 40, 3, 1):
        how = ro.ro_sampling(torch.full((n,), 0.9, device="cuda"), (torch.arange(n) % 90).int().cuda(),
                             torch.full((n,), 0.95, device="cuda"))
        token, kept = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
        logp = torch.zeros(n, device="cuda")
        ok(ctx, ro.ro_sample(ctx, dev[:n], how, u[:n].cuda(), token, logp, kept))
        ok(ctx, ro.ro_ctx_sync(ctx))
        base = base or (token, logp, kept)
        for got, want in zip((token, logp, kept), base):
            assert torch.equal(got, want[:n])
    check(ctx, x[:12], u[:12], temperature=0.9, top_k=kw["top_k"][:12], top_p=0.95)


def test_the_largest_vocabulary(ctx):
    x, u = rows(3, 393_216, F32, 1)
    check(ctx, x, u, top_p=[0.9, 1.0, 0.5])
    x, u = rows(2, 393_215, F32, 1)
    buf = torch.zeros(2, 393_216 + 7, device="cuda")
    buf[:, 3:3 + 393_215] = x.cuda()
    check(ctx, x, u, device=buf[:, 3:3 + 393_215], top_k=100)


def test_settings_out_of_range_are_recorded(ctx):
    x, u = rows(7, 500, F32, 5)
    dev = x.cuda()
    good = dict(temperature=[1.0] * 7, top_p=[0.9] * 7, min_p=[0.1] * 7, u=u.tolist())
    for name, bad in (("temperature", -1.0), ("temperature", math.nan), ("temperature", math.inf), ("top_p", 1.5), ("top_p", -0.1),
                      ("top_p", math.nan), ("min_p", 2.0), ("min_p", math.nan), ("u", 1.0), ("u", -0.1), ("u", math.nan)):
        a = {k: list(v) for k, v in good.items()}
        a[name][3] = bad
        f = {k: torch.tensor(v, dtype=F32).cuda() for k, v in a.items()}
        token, kept = (torch.zeros(7, dtype=torch.int32, device="cuda") for _ in range(2))
        logp = torch.zeros(7, device="cuda")
        ok(ctx, ro.ro_sample(ctx, dev, ro.ro_sampling(f["temperature"], None, f["top_p"], f["min_p"]), f["u"], token, logp, kept))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
        assert token[3].item() == NONE and kept[3].item() == 0 and logp[3].item() == -math.inf
        for r in (0, 1, 2, 4, 5, 6):
            assert token[r].item() == draw(x[r].double().numpy(), 1.0, 0, f["top_p"][r].item(), f["min_p"][r].item(),
                                           float(f["u"][r]))[0]
    ok(ctx, ro.ro_ctx_sync(ctx))


def test_on_another_stream_and_in_a_graph(ctx):
    side = torch.cuda.Stream()
    c2 = ro.ro_ctx_create(0, side, 1)
    try:
        x, u = rows(40, 50_000, BF16, 12)
        token, _, _ = check(ctx, x, u, temperature=0.8, top_p=0.9)
        dev, du = x.cuda(), u.cuda()
        how = ro.ro_sampling(torch.full((40,), 0.8, device="cuda"), None, torch.full((40,), 0.9, device="cuda"))
        out = torch.zeros(40, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ok(c2, ro.ro_sample(c2, dev, how, du, out))
        for _ in range(2):
            out.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, token)
        ok(c2, ro.ro_ctx_sync(c2))
    finally:
        ro.ro_ctx_destroy(c2)


def test_refusals(ctx):
    x, u = rows(3, 100, F32, 1)
    dev, du, token = x.cuda(), u.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        ro.ro_sample(ctx, dev.t(), None, du, token)
    with pytest.raises(ValueError):
        ro.ro_sample(ctx, dev, None, du[:2], token)
    with pytest.raises(ValueError):
        ro.ro_sample(ctx, dev, None, du, token[:2])
    with pytest.raises(ValueError):
        ro.ro_sample(ctx, dev.double(), None, du, token)
    with pytest.raises(ValueError):
        ro.ro_sample(ctx, dev, ro.ro_sampling(d_top_p=torch.ones(2, device="cuda")), du, token)
    big = torch.zeros(1, 393_217, device="cuda")
    assert ro.ro_sample(ctx, big, None, du, token) == ro.RO_E_OVERFLOW
    assert ro.ro_sample(ctx, dev[:, :0], None, du, token) == ro.RO_E_INVAL
    assert ro.ro_sample(ctx, dev[:0], None, du, token) == ro.RO_OK
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert token.tolist() == [0, 0, 0]
    ok(ctx, ro.ro_sample(ctx, dev, None, du, token))
    ok(ctx, ro.ro_ctx_sync(ctx))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows_of", [1, 30, 200])
def test_borders_of_the_candidates(ctx, dtype, rows_of):
    """Settings on either side of what is kept as a list of candidates: as many tokens as it holds, one more, twice as
    many, all of them equal but a few, far outliers and far lows."""
    V = 20_011
    x, u = rows(rows_of, V, dtype, 21, spread=1.0)
    for k in (383, 384, 385, 511, 512, 513, 704, 705, 1023, 1024, 1025, 2048, V - 1):
        check(ctx, x[:4], u[:4], top_k=k, top_p=[1.0, 0.9, 0.999, 0.5][:min(4, rows_of)])
    check(ctx, x[:4], u[:4], min_p=[0.2, 0.02, 0.002, 0.0002][:min(4, rows_of)], top_k=700)
    check(ctx, x[:4], u[:4], min_p=[0.2, 0.02, 0.002, 0.0002][:min(4, rows_of)], top_p=0.97)
    x[:, 100:1200] = x[:, :1]              # a run of equal ones, more than are listed
    check(ctx, x[:4], u[:4], top_k=50, min_p=0.001)
    check(ctx, x[:4], u[:4], top_p=0.3)
    x[:, 7] = 3e4
    check(ctx, x[:4], u[:4], top_k=50, top_p=0.999)
    x[:, ::5] = -6e4
    check(ctx, x[:4], u[:4], top_k=500, top_p=0.9, temperature=30.0)
    check(ctx, x[:4], u[:4], top_p=0.9999, temperature=3e4)


def test_sums_next_to_a_border(ctx):
    """Equal tokens whose running sum meets top-p's share exactly, and one step to either side."""
    n, V = 64, 40_960
    x = torch.full((1, V), -30.0)
    x[0, ::40] = 2.0                       # 1,024 equal ones
    for p in (0.25, 0.5, 0.125, 0.75):
        for q in (p, np.nextafter(np.float32(p), np.float32(0)), np.nextafter(np.float32(p), np.float32(1))):
            check(ctx, x, torch.tensor([0.999]), top_p=float(q), top_k=1024)
            check(ctx, x.expand(n, V)[:2], torch.tensor([0.2, 0.999]), top_p=float(q))


def test_many_rows_some_of_them_wide_in_a_graph(ctx):
    """Rows that few candidates decide and rows left to the second kernel, captured and replayed."""
    side = torch.cuda.Stream()
    c2 = ro.ro_ctx_create(0, side, 1)
    try:
        n, V = 320, 40_000
        x, u = rows(n, V, BF16, 31)
        dev, du = x.cuda(), u.cuda()
        p = torch.where(torch.arange(n) % 7 == 0, 0.97, 1.0)
        k = torch.where(torch.arange(n) % 7 == 0, 0, torch.where(torch.arange(n) % 11 == 0, 0, 40))
        token, logp, kept = check(ctx, x, u, top_p=p, top_k=k)
        how = ro.ro_sampling(None, k.int().cuda(), p.float().cuda())
        out, count = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
        share = torch.zeros(n, device="cuda")
        torch.cuda.synchronize()
        ok(c2, ro.ro_sample(c2, dev, how, du, out, share, count))
        ok(c2, ro.ro_ctx_sync(c2))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ok(c2, ro.ro_sample(c2, dev, how, du, out, share, count))
        for _ in range(3):
            for z in (out, share, count):
                z.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, token) and torch.equal(share, logp) and torch.equal(count, kept)
        ok(c2, ro.ro_ctx_sync(c2))
    finally:
        ro.ro_ctx_destroy(c2)


def test_outputs_that_share_memory_are_refused(ctx):
    x, u = rows(3, 100, F32, 1)
    dev, du = x.cuda(), u.cuda()
    ints, floats = torch.zeros(16, dtype=torch.int32, device="cuda"), torch.ones(16, device="cuda")
    how = ro.ro_sampling(floats[:3], ints[8:11], floats[3:6])
    for token, logp, kept in ((ints[8:11], None, None), (ints[10:13], None, None), (ints[:3], None, ints[2:5]),
                              (ints[:3], floats[2:5], None), (ints[:3], du, None), (ints[:3], dev[1, :3], None),
                              (ints[:3], dev.view(-1)[297:], None), (ints[:3], None, ints[6:9])):
        assert ro.ro_sample(ctx, dev, how, du, token, logp, kept) == ro.RO_E_INVAL
    ok(ctx, ro.ro_ctx_sync(ctx))
    ok(ctx, ro.ro_sample(ctx, dev, how, du, ints[:3], floats[6:9], ints[3:6]))
    ok(ctx, ro.ro_ctx_sync(ctx))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n", [3, 80])
@pytest.mark.parametrize("spread", [0.2, 1.5])
def test_wide_rows_of_all_settings(ctx, dtype, n, spread):
    """Rows that keep thousands of tokens, few of them and more than are worked on at a time: nuclei within top-k, cut
    shorter by min-p or not, borders between equal logits; calls one after the other."""
    V = 40_001
    for seed in (n, n + 1):
        x, u = rows(n, V, dtype, seed, spread)
        x[::7, 5000:9000] = x[::7, 4999:5000]      # borders among equal ones
        g = np.random.default_rng(seed)
        check(ctx, x, u, temperature=g.choice([0.7, 1.0, 2.0], n), top_k=g.choice([0, 0, 1500, 20_000, V - 1], n),
              top_p=g.choice([0.3, 0.9, 0.999, 1.0], n), min_p=g.choice([0.0, 0.0, 1e-4, 0.02], n))
