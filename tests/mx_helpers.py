"""Shared plumbing of the tests of the cache in 4 bits and of further eviction."""
from __future__ import annotations

import numpy as np
import torch

from oracle import mx_oracle as mxo
from tests import helpers as hp


def gauss(rng, *shape, dtype="bf16", size=1.0):
    """float32 array of Gaussian values that `dtype` holds exactly."""
    x = torch.from_numpy((rng.standard_normal(shape) * size).astype(np.float32))
    return (x.bfloat16().float() if dtype == "bf16" else x).numpy()


def prefix(lens):
    return np.concatenate(([0], np.cumsum(lens))).astype(np.int32)


def device(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda")


def cache(K, V, spare=0, fill=0xA5):
    """A packed cache of K and V in 4 bits on the device (stored by the oracle), with `spare` rows of `fill` behind it."""
    m = hp.mk()
    parts = [*mxo.store(K), *mxo.store(V)]
    return m.MxCache(*(device(np.concatenate((p, np.full((spare, p.shape[1]), fill, dtype=np.uint8)))) for p in parts))


def stored(K):
    """The values that K has in the cache, float64."""
    return mxo.values(*mxo.store(K))


def desc(B, H, d, dtype, n, P_max, g=1, prompt_len=None):
    m = hp.mk()
    return m.Desc(B=B, H=H, d=d, dtype=m.MASKKV_BF16 if dtype == "bf16" else m.MASKKV_F32, n_resp=n, P_max=P_max,
                  q_per_kv=0 if g == 1 else g, prompt_len=prompt_len)


# Error bounds, worst case, u = 2^-24 (half a step of fp32).  A logit is a sum of d products (exact for bf16): at most d roundings of
# partial sums, each of at most u times the sum S of the products' magnitudes, then the scale, the subtraction of a reference and
# the exponential (v_exp_f32: an ulp): 8 u times the largest magnitude among the terms, and 64 u for everything that is absolute.
U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}


def logit_error(Q, K, scale, *more):
    Q, K = np.abs(np.nan_to_num(np.asarray(Q, np.float64))), np.abs(np.asarray(K, np.float64))    # (NaN: of rows that do not count)
    S = Q @ K.T * scale
    top = max([S.max() if S.size else 0.0] + [np.abs(x).max() for x in more if np.size(x)])
    return U * ((Q.shape[1] + 4) * (S.max() if S.size else 0.0) + 8 * top + 64)


def check_attention(O, lse, Q, K, V, dtype, scale=None, tag=""):
    """O, lse (float64 arrays of the device's results) of queries Q over K, V against the oracle.

    A probability is off by twice a logit's error and, as the operand of the second product, by half a step of the dtype; the
    sums over the keys by a rounding a key; the result by half a step."""
    scale = 1.0 / np.sqrt(Q.shape[1]) if scale is None else scale
    ref, norm, mass = mxo.attend(Q, K, V, scale)
    e = logit_error(Q, K, scale, norm)
    keys = K.shape[0]
    bound = mass * (2 * e + 2 * (keys + 40) * U + HALF[dtype] * 1.02) + np.abs(ref) * HALF[dtype] * 1.02 + 1e-30
    off = np.abs(O - ref) / bound
    assert off.max() <= 1.0, f"{tag}: an output is {off.max():.2f} times its bound off"
    if lse is not None:
        far = np.abs(lse - norm).max()
        assert far <= 2 * e + (keys + 40) * U, f"{tag}: a normaliser is {far:.3e} off, {2 * e + (keys + 40) * U:.3e} allowed"


def check_weights(got, Q, K, lse, decay, before, scale=None, tag=""):
    scale = 1.0 / np.sqrt(Q.shape[1]) if scale is None else scale
    fresh = mxo.accumulate(Q, K, lse, scale=scale)
    want = fresh + (decay * before if decay else 0.0)
    finite = lse[np.isfinite(lse)]
    e = logit_error(Q, K, scale, finite)
    bound = fresh * (2 * e + (Q.shape[0] + 40) * U) + np.abs(want) * 4 * U + 1e-37
    off = np.abs(got - want) / bound
    assert off.size == 0 or off.max() <= 1.0, f"{tag}: a weight is {off.max():.2f} times its bound off"
