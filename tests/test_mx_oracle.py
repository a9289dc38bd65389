"""Pins of the oracle of the 4-bit cache and of further eviction (CPU): brute force and closed forms."""
import math

import numpy as np
import pytest

from oracle import mx_oracle as mxo


def test_every_stored_value_is_the_nearest_and_the_scale_the_smallest():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 64)) * np.exp2(rng.integers(-20, 20, (40, 1)))
    codes, scales = mxo.store(x)
    v = mxo.values(codes, scales)
    for r in range(40):
        for g in range(2):
            y, unit = x[r, 32 * g:32 * g + 32], 2.0 ** (int(scales[r, g]) - 127)
            assert np.abs(y).max() <= 6 * unit and np.abs(y).max() > 3 * unit
            grid = [s * z * unit for s in (1, -1) for z in mxo.SIZES]
            for a, b in zip(y, v[r, 32 * g:32 * g + 32]):
                assert abs(a - b) == min(abs(a - z) for z in grid)


def test_values_that_the_format_holds_come_back():
    sizes = np.array([s * z for s in (1, -1) for z in mxo.SIZES] * 2)          # 32 of them, 6 the largest
    for e in (-124, -30, 0, 7, 125):
        x = sizes[None] * 2.0 ** e
        codes, scales = mxo.store(x)
        assert scales.tolist() == [[e + 127]]
        assert np.array_equal(mxo.values(codes, scales), x)
        assert codes[0, :8].tolist() == [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] or x[0, 8] == 0.0


@pytest.mark.parametrize("value,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (0.2500001, 1)])
def test_ties_go_to_the_even_code(value, code):
    x = np.zeros((1, 32))
    x[0, 0], x[0, 1] = 6.0, value
    codes, scales = mxo.store(x)
    assert scales[0, 0] == 127 and codes[0, 0] == (7 | code << 4)


def test_edges_of_the_range_and_groups_that_are_no_numbers():
    x = np.zeros((6, 32))
    x[1, 3], x[2, 4] = np.nan, -np.inf
    x[3, 0] = 2.0 ** 128 * (1 - 2.0 ** -9)                                       # the largest bf16: beyond 6 * 2^125
    x[4, 0] = 2.0 ** -133                                                      # the smallest bf16
    x[5, 0] = 2.0 ** -125
    codes, scales = mxo.store(x)
    assert scales[:, 0].tolist() == [3, 255, 255, 252, 3, 3]
    assert codes[0].tolist() == [0] * 16 and codes[1].tolist() == [0] * 16
    v = mxo.values(codes, scales)
    assert np.isnan(v[1:3]).all()
    assert v[3, 0] == 6 * 2.0 ** 125 and v[4, 0] == 0.0 and v[5, 0] == 0.5 * 2.0 ** -124


def test_accumulate_sums_the_attention_that_attend_forms():
    rng = np.random.default_rng(2)
    Q, K, V = rng.standard_normal((5, 64)), rng.standard_normal((9, 64)), rng.standard_normal((9, 64))
    O, lse, mass = mxo.attend(Q, K, V)
    got = mxo.accumulate(Q, K, lse)
    assert abs(got.sum() - 5) < 1e-12                                          # rows of a softmax
    brute = [sum(math.exp(Q[i] @ K[j] / 8 - lse[i]) for i in range(5)) for j in range(9)]
    assert np.allclose(got, brute, rtol=1e-12)
    assert np.allclose(O[2], sum(math.exp(Q[2] @ K[j] / 8 - lse[2]) * V[j] for j in range(9)))
    assert (mass >= np.abs(O) - 1e-15).all()
    assert np.allclose(mxo.accumulate(Q, K, lse, 0.5, np.ones(9)), got + 0.5)
    lse[3] = np.inf
    assert np.allclose(mxo.accumulate(Q, K, lse).sum(), 4)


def test_stay_keeps_the_largest_and_breaks_ties_downwards():
    nan, inf = float("nan"), float("inf")
    assert mxo.stay([3, 1, 2, 3, 3], 2).tolist() == [0, 3]
    assert mxo.stay([0.0, -0.0, -1.0, 0.0], 2).tolist() == [0, 1]
    assert mxo.stay([nan, -inf, 1, nan, inf], 3).tolist() == [1, 2, 4]
    assert mxo.stay([nan, -inf, 1, nan, inf], 4).tolist() == [0, 1, 2, 4]
    assert mxo.stay([1, 2], 5).tolist() == [0, 1] and mxo.stay([1, 2], -3).tolist() == [] and mxo.stay([], 3).tolist() == []
