"""Float64 definitions of what surrounds the attention of an answer: rotary positions, masks among the response rows, tokens from logits.

Test infrastructure, written from the formulas; nothing here is shared with the library.
"""
import math

import numpy as np


def frequencies(width, base, scaling="plain", factor=1.0, trained=0.0, slow=1.0, fast=32.0):
    """Radians a position of each pair, and the amplitude."""
    out = []
    if scaling == "base" and width > 2:
        base = base * factor ** (width / (width - 2.0))
    for i in range(width // 2):
        f = base ** (-2.0 * i / width)
        if scaling == "linear":
            f = f / factor
        if scaling == "bands":
            turns = trained * f / (2.0 * math.pi)
            w = 1.0 if turns >= fast else 0.0 if turns <= slow else (turns - slow) / (fast - slow)
            f = f * (w + (1.0 - w) / factor)
        out.append(f)
    return np.array(out), 1.0 + 0.1 * math.log(factor) if scaling == "bands" else 1.0


def rotate(x, positions, freq, amplitude, width, layout):
    """x [..., T, d], positions [T] -> the rows turned, float64."""
    y = np.array(x, dtype=np.float64)
    half = width // 2
    for i in range(half):
        a, b = (i, i + half) if layout == "halves" else (2 * i, 2 * i + 1)
        angle = np.asarray(positions, dtype=np.float64) * freq[i]
        c, s = np.cos(angle), np.sin(angle)
        u, v = np.array(x[..., a], dtype=np.float64), np.array(x[..., b], dtype=np.float64)
        y[..., a], y[..., b] = amplitude * (u * c - v * s), amplitude * (v * c + u * s)
    return y


def tree(parents):
    """[n] -> [n, n]: whether row i sees row j."""
    n = len(parents)
    sees = np.zeros((n, n), dtype=bool)
    for i in range(n):
        if parents[i] < -1:
            continue
        j = i
        while True:
            sees[i, j] = True
            up = parents[j]
            if not 0 <= up < j or parents[up] < -1:
                break
            j = up
    return sees


def words(sees):
    """[..., n, n] -> the mask's words, uint32 [..., n, (n + 31) // 32]."""
    n = sees.shape[-1]
    out = np.zeros(sees.shape[:-1] + ((n + 31) // 32,), dtype=np.uint32)
    for j in range(n):
        out[..., j // 32] |= sees[..., j].astype(np.uint32) << np.uint32(j % 32)
    return out


def attend(Q, Kc, Vc, Kr, Vr, sees, scale=None):
    """Q [g, n, d] over cached rows and the response rows each query sees -> O [g, n, d], normalisers [g, n], sum_j a_ij |v_j|."""
    g, n, d = Q.shape
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    O, lse, mass = np.zeros((g, n, d)), np.full((g, n), -np.inf), np.zeros((g, n, d))
    for h in range(g):
        for i in range(n):
            K = np.concatenate((Kc, Kr[sees[i]])).astype(np.float64)
            V = np.concatenate((Vc, Vr[sees[i]])).astype(np.float64)
            if not len(K):
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                s = K @ Q[h, i].astype(np.float64) * scale
                top = s.max()
                p = np.exp(s - top)
                total = p.sum()
                O[h, i], mass[h, i] = (p / total) @ V, (p / total) @ np.abs(V)
                lse[h, i] = top + math.log(total) if total > 0 else np.nan
    return O, lse, mass


def sample(l, temperature, top_k, top_p, min_p, u):
    """One row -> token, prob, logprob, and how far the draw and the limit of top_p are from where they would come out otherwise,
    relative to the masses that decide them."""
    l = np.array(l, dtype=np.float64)
    l[np.isnan(l)] = -np.inf
    V = l.size
    top = l.max()
    if top == -np.inf:
        return -1, 0.0, -np.inf, 1.0
    if top == np.inf:
        l, top = np.where(l == np.inf, 0.0, -np.inf), 0.0
    logs = l - top - math.log(np.exp(l - top).sum())
    if not temperature > 0:
        at = int(np.argmax(l))
        return at, 1.0, logs[at], 1.0
    with np.errstate(invalid="ignore"):
        w = np.exp(np.where(l == -np.inf, -np.inf, (l - top) / float(temperature)))
    order = np.lexsort((np.arange(V), -l))
    stays = np.ones(V, dtype=bool)
    stays[order] = np.arange(V) < top_k if top_k > 0 else True
    margin = 1.0
    if top_p < 1:
        masses = np.where(stays[order], w[order], 0.0)
        upto = np.cumsum(masses)
        before = np.concatenate(([0.0], upto[:-1]))
        limit = float(top_p) * upto[-1]
        stays[order] &= (before < limit) | (np.arange(V) == 0)
        margin = np.abs(before[1:] - limit).min() / upto[-1] if V > 1 else 1.0
    if min_p > 0:
        stays &= w >= min(float(min_p), 1.0)
    stays &= w > 0
    kept = np.nonzero(stays)[0]
    upto = np.cumsum(w[kept])
    u = 1.0 - 2.0 ** -24 if not u < 1 else max(float(u), 0.0)
    target = u * upto[-1]
    at = min(int(np.searchsorted(upto, target, side="right")), kept.size - 1)
    margin = min(margin, np.abs(upto - target).min() / upto[-1])
    return int(kept[at]), w[kept[at]] / upto[-1], logs[kept[at]], margin
