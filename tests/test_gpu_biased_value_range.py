"""Values of any size under a cap: chunks over a bf16 cache, whose rows share one
reference for their weights, give what a running maximum gives."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2609_18703_gb300 as ro  # noqa: E402
from tests.test_gpu_biased import BF16, Cache, Case, _built, build, ctx, masks, ok  # noqa: E402,F401


def size(x, exponents):
    """bf16 times powers of two, without passing through other types' ranges."""
    return torch.ldexp(x.double(), torch.as_tensor(exponents, dtype=torch.int32)).to(BF16)


def near_cap(case, sign):
    """Products far beyond the cap."""
    case.q[:] = case.q.abs() * 4
    case.c.k[:] = (case.c.k.abs() + 2) * sign
    return case


@pytest.mark.parametrize("cap", [2.0, 5.0, 30.0, 50.0])
@pytest.mark.parametrize("exponent", [105, 90, -40, -105])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dim,page", [(64, 32), (128, 64)])
def test_all_values_far_from_one(ctx, cap, exponent, sign, dim, page):   # noqa: F811
    c = Cache([400, 90], 2, dim, page, BF16, 8, junk=0.0)
    c.v[:] = size(c.v, exponent)
    near_cap(Case(c, [90, 60], 4, cap=cap, scale=0.125), sign).check(ctx)


@pytest.mark.parametrize("cap", [5.0, 30.0, 50.0])
@pytest.mark.parametrize("form", [dict(), dict(docs=150), dict(window=70, sinks=3), dict(frame=40)])
def test_some_rows_and_columns_far_from_one(ctx, cap, form):   # noqa: F811
    """Values of every size among one another, scores from one end of the cap to the other; the next call as before."""
    lens, news = [700, 333, 40], [300, 333, 17]
    f = dict(form)
    first, until = masks(lens, news, f.pop("docs", 0), f.pop("frame", 0), 3, pads=0.1)
    usual = Case(Cache(lens, 2, 64, 16, BF16, 4, junk=0.0), news, 4, cap=cap, first=first, until=until, seed=4, **f)
    before = [x.clone() for x in usual.check(ctx)]
    c = Cache(lens, 2, 64, 16, BF16, 4, junk=0.0)
    g = np.random.default_rng(4)
    c.v[:] = size(c.v, g.choice([100, 0, -100], (1, 1, 1, 64)) * np.ones(tuple(c.v.shape)))   # by columns
    far = g.choice(c.k.shape[0], c.k.shape[0] // 2, replace=False)
    c.k[far] = c.k[far] * 40
    case = Case(c, news, 4, cap=cap, first=first, until=until, seed=4, **f)
    out, lse = [x.clone() for x in case.check(ctx)]
    again, lse2 = case.check(ctx)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    usual.call(ctx)
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert torch.equal(usual.out, before[0]) and torch.equal(usual.lse, before[1])


@pytest.mark.parametrize("cap", [30.0, 50.0])
@pytest.mark.parametrize("exponent", [100, -100])
@pytest.mark.parametrize("sign", [1, -1])
def test_long_caches_in_runs(ctx, cap, exponent, sign):   # noqa: F811
    """Pieces done again next to pieces that are not, joined; more pieces than the call before had, and fewer."""
    for news in ([70, 20], [700, 3], [40, 1]):
        c = Cache([9000, 700], 1, 64, 64, BF16, 4, junk=0.0)
        at = c.pages[:c.base[1]].long()[60:75]     # a thousand slots
        c.v[at] = size(c.v[at], exponent)
        case = Case(c, news, 4, cap=cap, scale=0.125)
        c.k[at] = (c.k[at].abs() + 2) * sign
        case.q[:] = case.q.abs() * 4
        case.check(ctx)


def test_in_a_graph_beside_other_calls(ctx):   # noqa: F811
    side = torch.cuda.Stream()
    c2 = ro.ro_ctx_create(0, side, 1)
    try:
        lens, news = [900, 333], [300, 200]
        c = Cache(lens, 2, 64, 16, BF16, 4, junk=0.0)
        c.v[:] = size(c.v, 100)
        case = near_cap(Case(c, news, 4, cap=50.0, scale=0.125), 1)
        want, want_lse = [x.clone() for x in case.check(ctx)]
        usual = Case(Cache([5000, 90], 2, 64, 16, BF16, 4, junk=0.0), [2000, 60], 4, cap=50.0)
        out, lse = [x.clone() for x in usual.check(ctx)]
        torch.cuda.synchronize()
        case.call(c2)
        ok(c2, ro.ro_ctx_sync(c2))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            case.call(c2)
        for _ in range(3):
            case.out.zero_()
            case.lse.zero_()
            usual.out.zero_()
            torch.cuda.synchronize()
            usual.call(c2)                         # more pieces: a larger workspace
            ok(c2, ro.ro_ctx_sync(c2))
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(case.out, want) and torch.equal(case.lse, want_lse)
            assert torch.equal(usual.out, out)
        ok(c2, ro.ro_ctx_sync(c2))
    finally:
        ro.ro_ctx_destroy(c2)
