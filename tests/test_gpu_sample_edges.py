"""Sampling where its kernels' choices lie: thresholds at zero, temperatures below
the normal numbers, rows split over one CTA or many, lists of candidates that are
just full.  Tokens and counts against the definition in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2609_18703_gb300 as ro  # noqa: E402
from tests.test_gpu_sample import BF16, F16, F32, _built, check, ctx, ok, rows  # noqa: E402,F401


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,V", [(1, 3), (1, 2051), (1, 70_001), (6, 1024), (320, 40_000)])
def test_largest_logit_of_zero_and_all_of_min_p(ctx, dtype, n, V):   # noqa: F811
    """Logits shifted by their largest, of which min-p of 1 keeps the largest alone: 0, -0 and several of either."""
    x, u = rows(n, V, dtype, V + n)
    x = -(x.float().abs() + 0.5).to(dtype)
    for r in range(n):
        x[r, r % V] = (0.0, -0.0)[r % 2]
        if r % 3 == 0:
            x[r, V - 1], x[r, V // 2] = -0.0, 0.0
    at = np.arange(n)
    temperature = np.array([1.0, 0.3, 7.0])[at % 3]
    check(ctx, x, u, min_p=1.0, temperature=temperature, top_p=np.array([1.0, 0.5, 0.999, 1.0])[at % 4])
    if n < 100:
        check(ctx, x, u, min_p=1.0)
        check(ctx, x, u, min_p=1.0, top_p=0.9)
        check(ctx, x, u, min_p=1.0, top_k=max(V - 1, 1), temperature=temperature)
        check(ctx, x, u, min_p=1.0, top_k=max(V - 1, 1), top_p=0.7)
