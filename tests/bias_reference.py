"""Biased attention from its definition, in 64 bits on the CPU, with the error
that 32-bit scores, one rounding of the weights and one of the output may leave."""
import math

import torch

from tests.step_reference import TINY, U


def seen(L, n, window, sinks, first=None, until=None):
    """[n, L]: which slots each of the last n tokens sees."""
    a = torch.arange(L - n, L)[:, None]
    j = torch.arange(L)[None]
    f = torch.zeros(n, 1, dtype=torch.int64) if first is None else first.long()[:, None]
    u = torch.zeros(n, 1, dtype=torch.int64) if until is None else until.long()[:, None]
    m = (j >= f) & (j < torch.maximum(a + 1, u)) & (f <= a) & (a >= 0)
    if window:
        m = m & ((j > a - window) | (j < f + sinks))
    return m


def attend(cache, s, q, scale, window, sinks, cap=0.0, slope=None, first=None, until=None):
    """q [n, heads, dim] of sequence s: out, lse, bounds of their errors."""
    n, H, D = q.shape
    L, K = cache.lens[s], cache.k.shape[1]
    dt = cache.k.dtype
    mask = seen(L, n, window, sinks, first, until)
    some = mask.any(1)
    used = mask.any(0)
    out = torch.zeros(n, H, D, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros_like(lse)
    if not bool(some.any()):
        return out, lse, tol, lse_tol
    apart = (torch.arange(L - n, L)[:, None] - torch.arange(L)[None]).abs().double()
    ks = cache.rows(cache.k, s).double()
    vs = cache.rows(cache.v, s).double()
    ks[:, ~used], vs[:, ~used] = 0, 0
    for h in range(H):
        k, v = ks[h // (H // K)], vs[h // (H // K)]
        x = scale * (q[:, h].double() @ k.T)
        # a 32-bit sum of D products and the scale: D + 4 roundings of the largest partial sum
        dx = (D + 4) * 2.0 ** -24 * abs(scale) * (q[:, h].double().abs() @ k.abs().T)
        if cap:
            # the argument and tanh are off by 2^-22 of them each at most; a flat cap forgets its argument's error
            dx = dx + 2.0 ** -22 * x.abs()
            lo, hi = torch.tanh((x - dx) / cap), torch.tanh((x + dx) / cap)
            x = cap * torch.tanh(x / cap)
            dx = torch.maximum(cap * hi - x, x - cap * lo) + 2.0 ** -22 * x.abs()
        if slope is not None:
            fall = float(slope[h]) * apart
            x = x - fall
            dx = dx + 2.0 ** -22 * fall.abs() + 2.0 ** -23 * x.abs()   # the slope in log2, the distance; one sum
        x = torch.where(mask, x, -math.inf)
        dx = torch.where(mask, dx, 0.0).amax(1, keepdim=True)
        z = torch.logsumexp(x, 1, keepdim=True)
        size = torch.where(mask, x.abs(), 0.0).amax(1, keepdim=True)
        p = torch.where(some[:, None], torch.exp(x - torch.where(some[:, None], z, 0.0)), 0.0)
        o = p @ v
        spread = p @ v.abs()
        small = TINY[dt] * torch.exp(x.amax(1, keepdim=True) - z).nan_to_num(0.0) * (mask.double() @ v.abs())
        # the weights' rounding, the exponentials' argument and 32 bits, the output's rounding
        rel = U[dt] + 2 * dx + 2.0 ** -22 * (size + 4) + 2.0 ** -20 + mask.sum(1, keepdim=True) * 2.0 ** -24
        out[:, h] = torch.where(some[:, None], o, 0.0)
        tol[:, h] = torch.where(some[:, None], (rel * spread + small) * 1.01 + U[dt] * o.abs() + TINY[dt], 0.0)
        lse[:, h] = z[:, 0]
        lse_tol[:, h] = (dx + 2.0 ** -22 * (z.abs() + size + 2))[:, 0]
    return out, lse, tol, torch.where(some[:, None], lse_tol, 0.0)
