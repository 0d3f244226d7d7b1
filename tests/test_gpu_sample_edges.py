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


SUBNORMAL = [2.0 ** -149, 1e-40, 1e-39, 4.2e-39, 4.3e-39, 1.2e-38]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,V", [(1, 1024), (6, 1000), (2, 40_001), (320, 40_000)])
def test_ties_at_the_smallest_temperatures(ctx, dtype, n, V):   # noqa: F811
    """Below the normal numbers only equal logits share a draw, and all of them do."""
    x, u = rows(n, V, dtype, V + n)
    for r in range(n):
        x[r, [r, V - 1 - r, V // 2][: 1 + (r + 1) % 3]] = 30.0
    at = np.arange(n)
    for temperature in SUBNORMAL if n < 100 else SUBNORMAL[2:3]:
        for top_p in (0.9, 0.4, 1.0):
            check(ctx, x, u, temperature=temperature, top_p=np.array([top_p, 0.6, top_p])[at % 3])
        if n < 100:
            check(ctx, x, u, temperature=temperature, top_k=V - 1, top_p=0.9)
            check(ctx, x, u, temperature=temperature, top_p=0.9, min_p=0.5)


@pytest.mark.parametrize("n,V", [(1, 900), (3, 3001), (2, 40_001), (200, 20_001)])
def test_logits_a_few_of_the_smallest_steps_apart(ctx, n, V):   # noqa: F811
    """Temperatures and differences of logits below the normal numbers: shares like any others."""
    g = np.random.default_rng(V)
    step = 2.0 ** -149
    x = torch.tensor(-g.integers(0, 400, (n, V)) * step, dtype=F32)
    u = torch.tensor(g.random(n), dtype=F32)
    for t in (7 * step, 64 * step) if n < 100 else (64 * step,):
        check(ctx, x, u, temperature=t)
        check(ctx, x, u, temperature=t, top_p=0.8)
        check(ctx, x, u, temperature=t, top_k=200, top_p=0.9)
        check(ctx, x, u, temperature=t, min_p=0.4)


@pytest.mark.parametrize("scale", [2.0 ** -126, 1e-30, 2.0 ** -64, 2.0 ** 64, 1e31, 1e37])
@pytest.mark.parametrize("n,V", [(3, 3001), (200, 20_001)])
def test_logits_and_temperatures_of_one_size(ctx, scale, n, V):   # noqa: F811
    """A row's draw is that of the same row times any number that leaves 32 bits' range alone."""
    x, u = rows(n, V, F32, 5)
    x = (x.double() * scale).float()
    check(ctx, x, u, temperature=scale, top_p=np.array([1.0, 0.9, 0.4])[np.arange(n) % 3])
    check(ctx, x, u, temperature=0.7 * scale, top_k=np.array([0, 60, 2000])[np.arange(n) % 3], min_p=0.001)
