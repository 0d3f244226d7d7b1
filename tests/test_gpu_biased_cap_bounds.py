"""The largest and smallest caps and ratios of scale and cap: right up to the
stated bounds on every kernel, refused beyond them."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2609_18703_gb300 as ro  # noqa: E402
from tests.test_gpu_biased import BF16, F16, Cache, Case, _built, ctx, ok  # noqa: E402,F401


@pytest.mark.parametrize("cap,scale", [(1e30, 0.125), (1e30, 2e-7), (1e-6, 0.125), (1e-6, 1e-6), (1e30, -0.125), (1e30, 0.0), (1e7, 1e-30)])
@pytest.mark.parametrize("news", [[1, 2], [90, 60]])
@pytest.mark.parametrize("dtype,page", [(BF16, 32), (F16, 32), (BF16, 5)])
def test_at_the_bounds(ctx, cap, scale, news, dtype, page):   # noqa: F811
    Case(Cache([500, 90], 2, 64, page, dtype, 8), news, 4, cap=cap, scale=scale).check(ctx)


@pytest.mark.parametrize("news", [[1, 2], [90, 60]])
def test_beyond_the_bounds(ctx, news):   # noqa: F811
    case = Case(Cache([500, 90], 2, 64, 32, BF16, 8), news, 4).device()
    for cap, scale in ((1.1e30, 0.125), (2.4e38, 0.125), (3.4e38, 1.0), (1e30, 1e-8), (1.0, 1e-38), (9e-7, 0.1), (1e-6, 1.1e24),
                       (1e30, -1e-8), (math.inf, 0.1), (math.nan, 0.1), (-1.0, 0.1)):
        case.scale, case.bias = scale, ro.ro_bias(cap)
        status = ro.ro_cache_attend_biased(ctx, case.cache, case.tok_base, max(news), case.len, 500, case.dq, scale, 0, 0, case.bias,
                                           case.out, case.lse)
        assert status == ro.RO_E_INVAL, (cap, scale)
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert bool((case.out == 9).all()) and bool((case.lse == 9).all())
