"""Scores millions from 0 over f16 caches: weights stay in f16's range, whatever
the kernel (single tokens, frames of a chunk, odd pages)."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2609_18703_gb300 as ro  # noqa: E402
from tests import slope_reference as ref  # noqa: E402
from tests.test_gpu_biased import BF16, F16, Cache, Case, _built, ctx, masks, ok, starts, within  # noqa: E402,F401


def check(ctx, case):   # noqa: F811
    case.device().call(ctx)
    ok(ctx, ro.ro_ctx_sync(ctx))
    t = starts(case.news)
    for s, n in enumerate(case.news):
        if n == 0:
            continue
        r = slice(t[s], t[s + 1])
        out, lse, tol, lse_tol = ref.attend(case.c, s, case.q[r], case.scale, case.window, case.sinks, case.cap, case.slope,
                                            None if case.first is None else case.first[r],
                                            None if case.until is None else case.until[r])
        within(case.out[r], out, tol)
        got, empty = case.lse[r].double().cpu(), torch.isinf(lse)
        assert torch.equal(torch.isinf(got) & (got < 0), empty)
        within(got[~empty], lse[~empty], lse_tol[~empty])


@pytest.mark.parametrize("slopes", [[1e5, 1e6, 3e7, 1e9], [-1e5, -1e6, -3e7, -1e9]])
@pytest.mark.parametrize("news", [[2, 1, 3], [130, 33, 300]])
@pytest.mark.parametrize("dtype,dim,page", [(F16, 64, 16), (F16, 128, 64), (F16, 64, 5), (BF16, 64, 16)])
def test_slopes_that_take_scores_far_from_zero(ctx, slopes, news, dtype, dim, page):   # noqa: F811
    """(Chunks: each frame is its sequence's whole cache, so that no slot lies ahead of all rows of a tile.)"""
    lens = [150, 700, 300]
    until = [L for L, n in zip(lens, news) for _ in range(n)]
    case = Case(Cache(lens, 2, dim, page, dtype, 5, junk=0.0), news, 4, until=until, seed=5)
    case.slope = torch.tensor(slopes)
    check(ctx, case)


@pytest.mark.parametrize("news", [[2, 1], [90, 40]])
@pytest.mark.parametrize("page", [16, 5])
def test_caps_that_leave_scores_far_from_zero(ctx, news, page):   # noqa: F811
    """Products of some 10^8 under a cap as large."""
    case = Case(Cache([300, 60], 2, 64, page, F16, 6, junk=0.0), news, 4, cap=1e8, scale=3e6, seed=6)
    check(ctx, case)
