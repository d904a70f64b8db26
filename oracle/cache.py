"""The 8-bit cache in numpy, from the definitions in include/attn.h: codes as the E4M3 values they stand for (float64), one power of two
for each 64 tokens of a head.  One token, one block, one head at a time."""
import math

import numpy as np

from .fp8 import round_to_e4m3

BLOCK = 64
LOWEST, HIGHEST = -100, 119


def exponent_for(amax):
    """The least e in [LOWEST, HIGHEST] with amax <= 448 * 2^e (HIGHEST if there is none)."""
    e = LOWEST
    while e < HIGHEST and amax > math.ldexp(448.0, e):
        e += 1
    return e


def quantise(x, e):
    """E4M3 values of x * 2^-e; infinities and what lies beyond become 448."""
    with np.errstate(invalid="ignore"):
        return round_to_e4m3(np.clip(np.asarray(x, dtype=np.float64) * 2.0 ** -e, -448.0, 448.0)).astype(np.float64)


class Cache:
    """K and V of one head of one sequence: values [capacity, d] and exponents [capacity / 64] each."""

    def __init__(self, capacity, d):
        self.values = [np.zeros((capacity, d)) for _ in range(2)]
        self.exponents = [np.zeros(capacity // BLOCK, dtype=int) for _ in range(2)]

    def append(self, length, *new):
        """new K and V [n, d]: the last n of `length` tokens."""
        for values, exponents, x in zip(self.values, self.exponents, new):
            x = np.asarray(x, dtype=np.float64)
            first = length - len(x)
            for blk in range(first // BLOCK, -(-length // BLOCK)) if len(x) else ():
                lo, hi = max(first, blk * BLOCK), min(length, (blk + 1) * BLOCK)
                piece = x[lo - first:hi - first]
                finite = np.abs(piece[np.isfinite(piece)])
                e = exponent_for(finite.max() if finite.size else 0.0)
                if lo > blk * BLOCK:                       # older tokens stand in front
                    e = max(e, int(exponents[blk]))
                    old = slice(blk * BLOCK, lo)
                    if e != exponents[blk]:
                        values[old] = quantise(values[old] * 2.0 ** (int(exponents[blk]) - e), 0)
                values[lo:hi] = quantise(piece, e)
                exponents[blk] = e

    def dequantised(self, which, length):
        scale = 2.0 ** self.exponents[which][np.arange(length) // BLOCK]
        return self.values[which][:length] * scale[:, None]


def scores(q, k, alpha, causal):
    """alpha q k^T of the newest len(q) queries with the hidden ones at -inf: query i sees tokens up to len(k) - len(q) + i."""
    s = alpha * (np.asarray(q, dtype=np.float64) @ k.T)
    if causal:
        hidden = np.arange(len(k))[None, :] > np.arange(len(q))[:, None] + len(k) - len(q)
        s = np.where(hidden, -np.inf, s)
    return s


def attend(q, k, v, alpha, causal):
    """O, LSE, and sum of P |v| (what errors of single probabilities are measured against); rows that see nothing: 0, -inf, 0."""
    n, d = q.shape
    O, lse, size = np.zeros((n, d)), np.full(n, -np.inf), np.zeros((n, d))
    if len(k) == 0:
        return O, lse, size
    s = scores(q, k, alpha, causal)
    for i in range(n):
        seen = ~np.isneginf(s[i])
        if not seen.any():
            continue
        m = s[i, seen].max()
        p = np.exp(s[i, seen] - m)
        lse[i] = m + np.log(p.sum())
        p /= p.sum()
        O[i], size[i] = p @ v[seen], p @ np.abs(v[seen])
    return O, lse, size


def weights(q, k, lse, alpha, causal):
    """What each token of k got from the queries q, whose logsumexp is lse; queries with -inf add nothing."""
    real = ~np.isneginf(lse)
    if len(k) == 0 or not real.any():
        return np.zeros(len(k))
    return np.exp(scores(q, k, alpha, causal)[real] - np.asarray(lse, dtype=np.float64)[real, None]).sum(0)


def kept(weights, length, budget, recent):
    """Positions that stay, ascending: the last `recent` and the largest weights before them, equal ones by position, NaN above all."""
    if length <= budget:
        return list(range(length))
    old = length - recent
    order = sorted(range(old), key=lambda t: (0, 0.0, t) if math.isnan(weights[t]) else (1, -float(weights[t]), t))
    return sorted(order[:budget - recent]) + list(range(old, length))


def gathered(cache, which, positions):
    """Values [n, d] and exponents per block of the tokens at `positions`, regrouped."""
    values, exponents = [], []
    for lo in range(0, len(positions), BLOCK):
        block = positions[lo:lo + BLOCK]
        source = [int(cache.exponents[which][t // BLOCK]) for t in block]
        e = max(source)
        exponents.append(e)
        for t, s in zip(block, source):
            values.append(quantise(cache.values[which][t] * 2.0 ** (s - e), 0))
    return np.array(values), exponents
