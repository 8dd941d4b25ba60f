"""The 4-bit cache format and the attention over it in float64, for the tests: numpy only."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EDGES = (GRID[1:] + GRID[:-1]) / 2
BF16_MAX = float(torch.finfo(torch.bfloat16).max)


def decode(data: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Values (float64) of packed rows [..., d / 2] with block scales [..., d / 32]."""
    code = np.stack((data & 15, data >> 4), -1).reshape(*data.shape[:-1], -1)
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    return v * np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=-1)


def rounded(x: np.ndarray) -> np.ndarray:
    """The values (float64) that rows of d channels become in the cache."""
    x = np.clip(np.where(np.isnan(x), 0.0, x.astype(np.float64)), -BF16_MAX, BF16_MAX)
    y = x.reshape(*x.shape[:-1], -1, 32)
    big = np.abs(y).max(-1, keepdims=True)
    e = np.maximum(np.frexp(big)[1] - 1 - 2, -125)
    e = np.where(big == 0, -125, e)
    a = np.abs(y) / np.exp2(e.astype(np.float64))
    lo = np.searchsorted(EDGES, a, side="left")    # on an edge: the lower grid point
    hi = np.searchsorted(EDGES, a, side="right")   # on an edge: the upper one
    code = np.where(lo % 2 == 0, lo, hi)           # of the two the even code
    return (np.sign(y) * GRID[code] * np.exp2(e.astype(np.float64))).reshape(x.shape)


def attention(q, k, v, limits, scale):
    """q [R, d], k / v [n, d] (float64), row r sees the first limits[r] tokens: outputs [R, d] and how far the kernel
    may be from them.

    Probabilities are rounded to bf16 (half a step, 2^-8) in the numerator and the denominator alike, so an output is
    off by at most 2^-8 times the weighted mean of |v - o| <= |v| + |o|, and then rounded to bf16 (2^-8 |o|).  A score
    is a sum of 128 exact products in float32: 130 roundings of at most 2^-24 of the products' magnitude; with the
    scale and the exponential (some 2^-22) that is a relative error of each probability, above and below."""
    s = (q @ k.T) * scale
    s = np.where(np.arange(k.shape[0])[None] < np.asarray(limits)[:, None], s, -np.inf)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o, mag = p @ v, p @ np.abs(v)
    e = (130 * 2.0 ** -24) * scale * (np.abs(q) @ np.abs(k).T).max(-1, keepdims=True) + 2.0 ** -20
    return o, 2.0 ** -8 * (mag + 2 * np.abs(o)) * (1 + 2.0 ** -7) + 2 * e * (mag + np.abs(o)) + 1e-30
