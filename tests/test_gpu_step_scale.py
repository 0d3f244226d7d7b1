"""A scale that passes 32 bits once it is taken to log2 is refused like one that
is not finite, with nothing written."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2609_18703_gb300 as ro  # noqa: E402
from tests.test_gpu_biased import BF16, Cache, Case, _built, ctx, ok  # noqa: E402,F401


@pytest.mark.parametrize("scale", [2.4e38, -3e38, math.inf, math.nan])
@pytest.mark.parametrize("news", [[1, 2], [90, 60]])
def test_scales_past_32_bits(ctx, news, scale):   # noqa: F811
    case = Case(Cache([500, 90], 2, 64, 32, BF16, 8), news, 4, cap=1e30).device()
    lens, score = max(case.c.lens), torch.full((2, 2, 500), 9.0, device="cuda")
    rows = (case.cache, case.tok_base, max(news), case.len)
    assert ro.ro_cache_attend_biased(ctx, *rows, lens, case.dq, scale, 0, 0, case.bias, case.out, case.lse) == ro.RO_E_INVAL
    assert ro.ro_cache_attend(ctx, *rows, lens, case.dq, scale, 0, 0, case.out, case.lse) == ro.RO_E_INVAL
    assert ro.ro_cache_weigh(ctx, *rows, case.dq, scale, 0, 0, case.lse, 0.5, None, score) == ro.RO_E_INVAL
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert bool((case.out == 9).all()) and bool((case.lse == 9).all()) and bool((score == 9).all())
