"""The definition of a draw, row by row in 64 bits on the CPU."""

import math

import numpy as np

LIMITS = 0.9999999e-30, 1.0000001e30    # of a temperature: 1e-30 and 1e30, rounded to 32 bits or not

def draw(x, u, T=1.0, k=0, p=1.0, q=0.0):
    """(token, logprob, kept_logprob, kept, distance): distance is how near the nearest decision was, relative to the sums."""
    x, u, T, p, q = np.asarray(x, np.float64), float(np.float32(u)), float(T), float(p), float(q)   # of rows' own: 32 bits already
    if u < 0:
        return -1, 0.0, 0.0, 0, 1.0
    if not (u < 1) or not (T == 0 or LIMITS[0] <= T <= LIMITS[1]) or not 0 <= p <= 1 or not 0 <= q <= 1 or np.isnan(x).any() or (x == np.inf).any():
        return -1, math.nan, math.nan, 0, 1.0
    m = x.max()
    if m == -np.inf:
        return -1, -math.inf, -math.inf, 0, 1.0
    if T == 0:
        return int(np.argmax(x)), 0.0, 0.0, 1, 1.0
    w = np.exp((x - m) / T)
    order = np.argsort(-x, kind="stable")
    there = int((x > -np.inf).sum())
    K = min(k, there) if k > 0 else there
    sums, near = np.cumsum(w[order]), 1.0
    L = K
    if p < 1:
        B = p * sums[K - 1]
        L = min(K, int(np.searchsorted(sums[:K], B)) + 1)
        off = np.abs(sums[:K] / B - 1) if B > 0 else np.ones(1)
        near = off[off > 0].min() if (off > 0).any() else 1.0     # equal to the border: whole weights, whose sums are exact
    L = max(1, min(L, int((w[order[:L]] >= q).sum())))
    kept = np.zeros(len(x), bool)
    kept[order[:L]] = True
    run = np.cumsum(np.where(kept, w, 0.0))
    C = run[-1]
    token = int(np.searchsorted(run, u * C, side="right"))
    if u > 0:
        near = min(near, np.abs(run[kept] / (u * C) - 1).min())
    z = (x[token] - m) / T
    return token, z - math.log(w.sum()), z - math.log(C), L, near
