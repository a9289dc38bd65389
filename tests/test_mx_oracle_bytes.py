"""The bytes of the oracle's 4-bit cache, written out (CPU): which half of a byte an element is in, its sign, -0 and the scale."""
import numpy as np
import pytest

from oracle import mx_oracle as mxo

# 0, 0.5, 1, 1.5, 2, 3, 4, 6 and then the same with a minus, twice: codes 0 .. 15, the even element in the low four bits
BYTES = [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] * 2
VALUES = [s * z for s in (1.0, -1.0) for z in (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)] * 2


@pytest.mark.parametrize("e", [-124, -30, 0, 7, 125])
def test_the_packed_bytes_of_all_sixteen_codes(e):
    x = np.array([VALUES]) * 2.0 ** e
    codes, scales = mxo.store(x)
    assert codes.dtype == scales.dtype == np.uint8
    assert codes.tolist() == [BYTES] and scales.tolist() == [[e + 127]]


def test_the_values_of_given_bytes():
    codes = np.array([BYTES + BYTES[::-1]], dtype=np.uint8)
    v = mxo.values(codes, np.array([[127, 130]], dtype=np.uint8))
    assert v[0, :32].tolist() == VALUES
    back = [VALUES[2 * i + half] * 8.0 for i in reversed(range(16)) for half in (0, 1)]
    assert v[0, 32:].tolist() == back
    assert np.signbit(v[0, 8]) and not np.signbit(v[0, 0])                 # -0 and 0


def test_scales_belong_to_32_neighbours_in_their_order():
    x = np.concatenate((np.full(32, 6.0), np.full(32, -0.75), np.zeros(32), np.full(32, 192.0)))[None]
    codes, scales = mxo.store(x)
    assert scales.tolist() == [[127, 124, 3, 132]]
    assert codes.tolist() == [[0x77] * 16 + [0xFF] * 16 + [0x00] * 16 + [0x77] * 16]
