"""Float64 CPU oracle of the cache in 4 bits and of further eviction from a packed cache.  TEST INFRASTRUCTURE ONLY.

Plain definitions, one head at a time, as in ``maskkv_oracle``; no code shared with the HIP path.

* A group of 32 neighbours along the head dimension is stored with the smallest power of two 2^e for which no element is
  larger than 6 * 2^e (-124 <= e <= 125), and every element as the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e, ties to the
  value of even number in that list; what is beyond 6 * 2^125 becomes that, a group with a NaN or an infinity stands for NaN.
* The attention of a step over [cached rows ; response rows], and what of it each cached row gets.
* The rows of largest accumulated weight.
"""
from __future__ import annotations

import math

import numpy as np

SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GROUP = 32


def store(x):
    """Rows [n, d] -> codes uint8 [n, d/2] (even element in the low four bits) and scale bytes uint8 [n, d/32]."""
    with np.errstate(invalid="ignore"):                # (NaN of any kind)
        x = np.asarray(x, dtype=np.float64)
    n, d = x.shape
    codes, scales = np.zeros((n, d), dtype=np.uint8), np.zeros((n, d // GROUP), dtype=np.uint8)
    groups = x.reshape(n, d // GROUP, GROUP)
    finite = np.isfinite(groups).all(axis=2)
    scales[~finite] = 255
    most = np.where(finite, np.abs(np.where(np.isfinite(groups), groups, 0.0)).max(axis=2), 0.0)
    e = np.full(most.shape, -124)
    for step in range(-124, 126):                       # the smallest that holds the largest element
        e = np.where(most > 6.0 * math.ldexp(1.0, step), min(step + 1, 125), e)
    scales[finite] = (e + 127)[finite].astype(np.uint8)
    size = np.abs(np.where(finite[..., None], groups, 0.0)) / np.ldexp(1.0, e)[..., None]
    best, far = np.zeros(size.shape, dtype=np.uint8), np.full(size.shape, np.inf)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):               # the even ones first: they keep a tie
        gap = np.abs(size - SIZES[code])
        best = np.where(gap < far, code, best).astype(np.uint8)
        far = np.minimum(gap, far)
    sign = np.where(finite[..., None], np.signbit(groups), False).astype(np.uint8)
    codes = (best | sign << 3).reshape(n, d)
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8), scales


def values(codes, scales):
    """What stored rows stand for: float64 [n, d]."""
    codes = np.asarray(codes)
    n, half = codes.shape
    flat = np.empty((n, 2 * half), dtype=np.int64)
    flat[:, 0::2], flat[:, 1::2] = codes & 15, codes >> 4
    x = np.asarray(SIZES)[flat & 7] * np.where(flat & 8, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, np.asarray(scales, dtype=np.int64) - 127))
    return x * np.repeat(unit, GROUP, axis=1)


def attend(Q, K, V, scale=None):
    """Q [n, d], K, V [keys, d] -> O [n, d], natural-log normalisers [n], and sum_j a_ij |v_j| [n, d] (for error bounds)."""
    Q, K, V = (np.asarray(a, dtype=np.float64) for a in (Q, K, V))
    s = Q @ K.T * (1.0 / math.sqrt(Q.shape[1]) if scale is None else scale)
    top = s.max(axis=1, keepdims=True)
    p = np.exp(s - top)
    total = p.sum(axis=1, keepdims=True)
    p /= total
    return p @ V, (top + np.log(total))[:, 0], p @ np.abs(V)


def accumulate(Q, K, lse, decay=0.0, before=None, scale=None):
    """What each row of K gets from the queries with the given normalisers, on top of decay * before."""
    Q, K, lse = (np.asarray(a, dtype=np.float64) for a in (Q, K, lse))
    voting = lse != np.inf                              # the others add nothing, whatever they hold
    s = Q[voting] @ K.T * (1.0 / math.sqrt(Q.shape[1]) if scale is None else scale)
    got = np.exp(s - lse[voting, None]).sum(axis=0)
    return got if decay == 0.0 else decay * np.asarray(before, dtype=np.float64) + got


def stay(weights, budget):
    """The rows of one head that stay, ascending: the largest weights, ties to the lower row, NaN below every number."""
    w = np.asarray(weights, dtype=np.float64)
    k = min(max(int(budget), 0), w.shape[0])
    order = sorted(range(w.shape[0]), key=lambda r: (1, 0.0, r) if math.isnan(w[r]) else (0, -w[r], r))
    return np.array(sorted(order[:k]), dtype=np.int64)
