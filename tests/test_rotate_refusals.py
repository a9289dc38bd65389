"""What maskkv_rotate and maskkv_rotary_frequencies refuse or take at the edges of their arguments (CPU: the pointers are fake, and no call has rows to turn)."""
import math

import pytest

from tests.test_decode_refusals import F, desc, error, mk, rotate, view  # noqa: F401  (mk: a fixture)


@pytest.mark.parametrize("freq", [1e299, -1e299, math.ldexp(1.0, 993), 1.7e308, -1.7e308])
def test_a_frequency_whose_farthest_angle_is_no_number(mk, freq):
    """Positions reach 2^31: the angle would be infinite there, and its sine NaN."""
    r = mk.maskkv_rotary_frequencies(64)
    r.freq[5] = freq
    assert rotate(mk, rotary=r, lens=[0]) == 1 and "finite" in error(mk)
    r.freq[5] = math.copysign(math.ldexp(1.0, 992), freq)
    assert rotate(mk, rotary=r, lens=[0]) == 0


def test_frequencies_that_are_given_out_are_taken(mk):
    for base in (1e-290, 1e-300, 1e-305, 1e-307, 1e300):
        try:
            r = mk.maskkv_rotary_frequencies(64, mk.ROTARY_HALVES, base)
        except mk.MaskKVError as e:
            assert e.status == 1 and "range" in str(e)
            continue
        assert rotate(mk, rotary=r, lens=[0]) == 0
    with pytest.raises(mk.MaskKVError):
        mk.maskkv_rotary_frequencies(64, mk.ROTARY_HALVES, 1e-318)


def test_a_view_of_one_token_or_one_head_is_itself_whatever_its_stride(mk):
    """In place, a row a head: the stride between tokens that there are not says nothing, and likewise that between heads."""
    def strides(h, t):
        v = view(mk)
        v.stride_h, v.stride_t = h, t
        return v

    assert rotate(mk, n=1, lens=[0], Q=strides(64, 64), Q_out=strides(64, 128)) == 0
    assert rotate(mk, desc(mk, H=1), n=8, lens=[0], Q=strides(512, 64), Q_out=strides(4096, 64)) == 0
    assert rotate(mk, n=2, lens=[0], Q=strides(64, 64), Q_out=strides(64, 128)) == 1 and "same view" in error(mk)
    assert rotate(mk, desc(mk, q_per_kv=2, H=1), n=1, lens=[0], Q=strides(512, 64), Q_out=strides(4096, 64)) == 1 and "same view" in error(mk)
