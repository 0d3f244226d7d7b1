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


@pytest.mark.parametrize("dtype,V", [(BF16, 131_072), (F32, 40_001), (F16, 65_539)])
def test_row_counts_that_split_rows_otherwise_draw_alike(ctx, dtype, V):   # noqa: F811
    """Rows of several CTAs or one, decided by candidates, queued or wide from the start: the same draws."""
    most = 300
    x, u = rows(most, V, dtype, 77)
    at = torch.arange(most)
    temperature = torch.tensor([1.0, 0.7, 1.3, 2.0])[at % 4]
    top_k = torch.tensor([0, 50, 0, 0, 900, 0, V - 1])[at % 7].int()
    top_p = torch.tensor([1.0, 0.9, 0.95, 0.5, 1.0])[at % 5]
    min_p = torch.tensor([0.0, 0.0, 0.02])[at % 3]
    dev, du = x.cuda(), u.cuda()
    settings = [z.cuda() for z in (temperature, top_k, top_p, min_p)]
    base = None
    for n in (300, 160, 40, 12, 3, 1):
        how = ro.ro_sampling(*[z[:n].clone() for z in settings])
        token, kept = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        logp = torch.full((n,), 7.0, device="cuda")
        ok(ctx, ro.ro_sample(ctx, dev[:n], how, du[:n].clone(), token, logp, kept))
        ok(ctx, ro.ro_ctx_sync(ctx))
        base = base or (token, logp, kept)
        for got, want in zip((token, logp, kept), base):
            assert torch.equal(got, want[:n])
    check(ctx, x[:21], u[:21], temperature=temperature[:21], top_k=top_k[:21], top_p=top_p[:21], min_p=min_p[:21])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n", [1, 30, 200])
def test_borders_of_the_candidates_in_every_row(ctx, dtype, n):   # noqa: F811
    """Each row at another border of the lists of candidates, a CTA or a cluster a row, queued or not."""
    V = 40_011
    x, u = rows(n, V, dtype, 21, spread=1.0)
    ks = (383, 384, 385, 511, 512, 513, 704, 705, 1023, 1024, 1025, 2048, V - 1)
    at = np.arange(n)
    pick = lambda v, by=1: np.array(v)[at // by % len(v)]   # noqa: E731
    for shift in range(0, 13, 4) if n == 1 else (0,):
        check(ctx, x, u, top_k=pick(ks[shift:] + ks[:shift]), top_p=pick([1.0, 0.9, 0.999, 0.5], 13))
    check(ctx, x, u, min_p=pick([0.2, 0.02, 0.002, 0.0002]), top_p=pick([1.0, 0.97], 4), top_k=pick([700, 0], 8))
    check(ctx, x, u, top_p=pick([0.05, 0.2, 0.4, 0.6, 0.9]), temperature=pick([1.0, 0.5], 5))
    x[:, 100:1200] = x[:, :1]              # a run of equal ones, more than are listed
    check(ctx, x, u, top_k=pick([50, 0, 1100]), top_p=pick([1.0, 0.3], 3), min_p=pick([0.001, 0.0], 6))
    x[:, 7] = 3e4
    x[:, ::5] = -6e4
    check(ctx, x, u, top_k=pick([50, 500, 0]), top_p=pick([0.999, 0.9, 0.9999], 3), temperature=pick([1.0, 30.0, 3e4], 9))


@pytest.mark.parametrize("dtype,V", [(BF16, 131_072), (F32, 100_003)])
@pytest.mark.parametrize("spread", [0.01, 0.5, 3.0])
def test_numbers_next_to_the_borders_of_tokens(ctx, dtype, V, spread):   # noqa: F811
    """u right below, on and above a token's share of the running sum, sums from some hundred to V: draws by the
    definition, and the same of one row alone, of a few and of many."""
    most = 200
    x, _ = rows(most, V, dtype, 7, spread)
    g = np.random.default_rng(V)
    w = np.exp(x.double().numpy() - x.double().numpy().max(1, keepdims=True))
    runs = np.cumsum(w, 1)
    at = g.integers(V // 2, V, most)
    u = (runs[np.arange(most), at] / runs[:, -1]).astype(np.float32)
    u = torch.tensor(np.minimum(u + np.spacing(u) * g.integers(-1, 2, most), 1 - 2.0 ** -24).astype(np.float32))
    dev = x.cuda()
    token, logp, _ = check(ctx, x, u, device=dev)
    for n in (40, 1):
        out, share = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
        ok(ctx, ro.ro_sample(ctx, dev[:n], None, u[:n].cuda(), out, share))
        ok(ctx, ro.ro_ctx_sync(ctx))
        assert torch.equal(out, token[:n]) and torch.equal(share, logp[:n])
