"""Rotary positions and the paged cache, fp64.  Test infrastructure only.

Written from the definitions in include/logquant.h: rows are kept as lists of what every token came with, places by the
documented index formulas, angles as complex numbers, the tokens that stay by sorting.
"""
import numpy as np

from .cache8 import kperm


def frequencies(dims, base=10000.0, stretch=1.0, original=0.0, slow=1.0, fast=32.0):
    f = base ** (-np.arange(0, dims, 2) / dims)
    if original <= 0:
        return f / stretch
    turns = original * f / (2 * np.pi)
    w = np.clip((turns - slow) / (fast - slow), 0, 1)
    return w * f + (1 - w) * f / stretch


def partners(dims, interleaved):
    """Channels of the first and second halves of all pairs."""
    i = np.arange(dims // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)


def rotate(x, positions, freq, interleaved=False, factor=1.0):
    """x [..][L][d] turned by positions [L]."""
    x = np.array(x, np.float64)
    freq = np.asarray(freq, np.float64)
    one, two = partners(2 * len(freq), interleaved)
    z = (x[..., one] + 1j * x[..., two]) * (factor * np.exp(1j * np.asarray(positions, np.float64)[:, None] * freq))
    x[..., one], x[..., two] = z.real, z.imag
    return x


def scores(q, K, scale, softcap=0.0, slopes=None, window=0):
    """Scores [g][n] of queries q [g][d] over keys K [n][d]; -inf where a token gets no weight."""
    n = len(K)
    s = scale * (q @ K.T)
    if softcap > 0:
        s = softcap * np.tanh(s / softcap)
    ahead = n - 1 - np.arange(n)
    if slopes is not None:
        s = s - np.asarray(slopes, np.float64)[:, None] * ahead
    return np.where(ahead < window, s, -np.inf) if window > 0 else s


def probabilities(s):
    p = np.exp(s - s.max(-1, keepdims=True))
    return p / p.sum(-1, keepdims=True)


def kept(weights, keep, recent):
    """Tokens that stay of those with these weights, in order."""
    n = len(weights)
    if n <= keep:
        return np.arange(n)
    old = sorted(range(n - recent), key=lambda t: (-weights[t], t))[:keep - recent]
    return np.array(sorted(old) + list(range(n - recent, n)), dtype=np.int64)


def page_index(which, g, h, t, c, Hkv, page, d):
    """Index of (token t of the page, channel c) of kv head h in page g of a pool."""
    if which == "k":
        return ((((g * Hkv + h) * (page // 16) + t // 16) * (d // 32) + c // 32) * 64 + 16 * ((c % 32) // 8) + t % 16) * 8 + c % 8
    k = kperm(t % 32)
    return ((((g * Hkv + h) * (page // 32) + t // 32) * (d // 16) + c // 16) * 64 + 16 * (k // 8) + c % 16) * 8 + k % 8
