"""Attention with distance biases from its definition, in 64 bits on the CPU, with
a bound for every slot's own score: what a far slot's 32-bit score may be off
says nothing about a near one's."""
import math

import torch

from tests.bias_reference import seen
from tests.step_reference import TINY, U


def attend(cache, s, q, scale, window, sinks, cap=0.0, slope=None, first=None, until=None):
    """q [n, heads, dim] of sequence s: out, lse, bounds of their errors."""
    n, H, D = q.shape
    L, K = cache.lens[s], cache.k.shape[1]
    dt = cache.k.dtype
    mask = seen(L, n, window, sinks, first, until)
    some, used = mask.any(1), mask.any(0)
    out, tol = (torch.zeros(n, H, D, dtype=torch.float64) for _ in range(2))
    lse, lse_tol = torch.full((n, H), -math.inf, dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64)
    apart = (torch.arange(L - n, L)[:, None] - torch.arange(L)[None]).abs().double()
    ks, vs = cache.rows(cache.k, s).double(), cache.rows(cache.v, s).double()
    ks[:, ~used], vs[:, ~used] = 0, 0
    only = lambda x, other: torch.where(mask, x, other)   # noqa: E731
    for h in range(H):
        k, v = ks[h // (H // K)], vs[h // (H // K)]
        x = scale * (q[:, h].double() @ k.T)
        # a 32-bit sum of D products and the scale (twice, as it goes to log2): D + 5 roundings of the largest partial sum
        dx = (D + 5) * 2.0 ** -24 * abs(scale) * (q[:, h].double().abs() @ k.abs().T)
        if cap:   # the argument and tanh, 2^-22 each; a flat cap forgets its argument's error
            dx = dx + 2.0 ** -22 * x.abs()
            lo, hi = torch.tanh((x - dx) / cap), torch.tanh((x + dx) / cap)
            x = cap * torch.tanh(x / cap)
            dx = torch.maximum(cap * hi - x, x - cap * lo) + 2.0 ** -22 * x.abs()
        fall = torch.zeros_like(apart) if slope is None else float(slope[h]) * apart
        x = x - fall
        top = only(x, -math.inf).amax(1, keepdim=True).nan_to_num(neginf=0.0)
        # the slope in log2 (constant, product), one sum; its distance from the running maximum, which may lag by 2^8
        dx = dx + 2.0 ** -23 * fall.abs() + 2.0 ** -24 * x.abs() + 2.0 ** -23 * ((x - top).abs() + 8) + 2.0 ** -22
        x = only(x, -math.inf)
        z = torch.logsumexp(x, 1, keepdim=True)
        up, down = torch.logsumexp(only(x + dx, -math.inf), 1, keepdim=True), torch.logsumexp(only(x - dx, -math.inf), 1, keepdim=True)
        some_h = some[:, None]
        dz = torch.where(some_h, torch.maximum(up - z, z - down), 0.0) + mask.sum(1, keepdim=True) * 2.0 ** -24
        zero = torch.where(some_h, z, 0.0)
        p = torch.exp(x - zero)
        # each weight: its score, its rounding to the cache's type, the sum that it is divided by
        most = torch.exp(only(x - zero + dx + dz, -math.inf)) * (1 + U[dt])
        o = p @ v
        small = TINY[dt] * torch.where(some_h, torch.exp(top - zero), 0.0) * (mask.double() @ v.abs())
        off = (most - p) @ v.abs() + small
        out[:, h] = torch.where(some_h, o, 0.0)
        tol[:, h] = torch.where(some_h, off * 1.01 + U[dt] * (o.abs() + off) + TINY[dt], 0.0)
        lse[:, h] = z[:, 0]
        lse_tol[:, h] = torch.where(some, (dz + 2.0 ** -22 * (zero.abs() + top.abs() + 2))[:, 0], 0.0)
    return out, lse, tol, lse_tol
