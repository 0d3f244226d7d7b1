"""The model-step operators from their definitions, in 64 bits on the CPU, with
the error that 32-bit sums and one rounding to the type may leave."""
import math

import numpy as np
import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}   # one rounding, relative
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}   # half the smallest f16 step


def turn(x, pos, pairs, base, interleaved, inverse=False):
    """x [tokens, heads, dim] in 64 bits, turned."""
    y = x.double().clone()
    R, p = sum(pairs), 0
    for axis, width in enumerate(pairs):
        for _ in range(width):
            theta = pos[:, axis].double() * base ** (-p / R)
            c, s = torch.cos(theta)[:, None], torch.sin(theta)[:, None] * (-1 if inverse else 1)
            i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + R)
            a, b = x[..., i].double(), x[..., j].double()
            y[..., i], y[..., j] = a * c - b * s, b * c + a * s
            p += 1
    return y


class Cache:
    """A paged cache with its page lists, made on the CPU, mirrored on the GPU by device()."""

    def __init__(self, lens, heads, dim, page, dtype, seed, spare=3, junk=float("nan")):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page = list(lens), page
        held = [-(-L // page) for L in lens]
        n = sum(held) + spare
        self.k = torch.full((n, heads, page, dim), junk, dtype=torch.float64).to(dtype)
        self.v = self.k.clone()
        order = torch.randperm(n, generator=g)
        self.base = np.concatenate([[0], np.cumsum(held)]).astype(np.int64)
        self.pages = order[: sum(held)].int()
        self.free = order[sum(held):].int()
        for s, L in enumerate(lens):
            for j in range(0, L, page):
                m = min(page, L - j)
                at = int(self.pages[self.base[s] + j // page])
                self.k[at, :, :m] = torch.randn(heads, m, dim, generator=g).to(dtype)
                self.v[at, :, :m] = torch.randn(heads, m, dim, generator=g).to(dtype)

    def rows(self, pool, s, n=None):
        """[heads, n, dim] of a sequence's first n slots (its length)."""
        n = self.lens[s] if n is None else n
        j = np.arange(n)
        page = self.pages[self.base[s] + j // self.page].long()
        return pool[page, :, torch.as_tensor(j % self.page)].transpose(0, 1)


def seen(L, n, window, sinks):
    a = torch.arange(L - n, L)[:, None]
    j = torch.arange(L)[None]
    m = j <= a
    if window:
        m = m & ((j > a - window) | (j < sinks))
    return m


def attend(cache, s, q, scale, window, sinks):
    """q [n, heads, dim] of sequence s: out, lse, bounds of their errors."""
    n, H, D = q.shape
    L, K = cache.lens[s], cache.k.shape[1]
    dt = cache.k.dtype
    mask = seen(L, n, window, sinks)
    out = torch.zeros(n, H, D, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros_like(lse)
    ks, vs = cache.rows(cache.k, s).double(), cache.rows(cache.v, s).double()
    for h in range(H):
        k, v = ks[h // (H // K)], vs[h // (H // K)]
        for t in range(n):
            see = mask[t]
            if not bool(see.any()):
                continue
            x = scale * (k[see] @ q[t, h].double())
            # a 32-bit sum of D products, then the scale: D + 4 roundings of the largest partial sum
            dx = (D + 4) * 2.0 ** -24 * float((abs(scale) * (k[see].abs() @ q[t, h].double().abs())).max())
            p = torch.softmax(x, 0)
            lse[t, h] = torch.logsumexp(x, 0)
            lse_tol[t, h] = dx + 2.0 ** -22 * (abs(float(lse[t, h])) + float(x.abs().max()) + 2)
            out[t, h] = p @ v[see]
            spread = p @ v[see].abs()
            small = TINY[dt] * float(torch.exp(x.max() - lse[t, h])) * v[see].abs().sum(0)
            # the weights' rounding, the exponentials' and sums' 32 bits, the output's rounding
            rel = U[dt] + 2 * dx + 2.0 ** -20 + int(see.sum()) * 2.0 ** -24
            tol[t, h] = (rel * spread + small) * 1.01 + U[dt] * out[t, h].abs() + TINY[dt]
    return out, lse, tol, lse_tol


def weigh(cache, s, q, scale, window, sinks, lse, decay, past):
    """[heads, L] scores of sequence s and the bound of their error."""
    n, H, D = q.shape
    L, K = cache.lens[s], cache.k.shape[1]
    mask = seen(L, n, window, sinks)
    ks = cache.rows(cache.k, s).double()
    score = torch.zeros(K, L, dtype=torch.float64)
    old = max(L - n, 0)
    score[:, :old] = decay * past[:, :old].double()
    tol = score.abs() * 2.0 ** -22
    for h in range(H):
        k = ks[h // (H // K)]
        for t in range(n):
            if not bool(mask[t].any()):
                continue
            x = scale * (k @ q[t, h].double())
            big = abs(scale) * (k.abs() @ q[t, h].double().abs())
            w = torch.where(mask[t], torch.exp(x - float(lse[t, h])), torch.zeros(()).double())
            score[h // (H // K)] += w
            tol[h // (H // K)] += w * ((D + 4) * 2.0 ** -24 * big + 2.0 ** -21 * (2 + abs(float(lse[t, h])) + x.abs())
                                       + n * H * 2.0 ** -24)
    return score, tol


def evict(L, score, budget, sinks, recent):
    """Kept slots of one head (scores of its L slots)."""
    if L <= budget:
        return np.arange(L)
    x = np.asarray(score[:L], np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    nan = np.isnan(np.asarray(score[:L], np.float64))
    lo, hi = sinks, L - recent
    order = np.lexsort((np.arange(lo, hi), nan[lo:hi], -x[lo:hi]))[: budget - sinks - recent] + lo
    return np.sort(np.concatenate([np.arange(lo), order, np.arange(hi, L)])).astype(np.int64)
