"""What maskkv_rotate and maskkv_rotary_frequencies refuse or take at the edges of their arguments (CPU: the pointers are fake, and no call has rows to turn)."""
import ctypes as ct
import math

import numpy as np
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
    assert rotate(mk, n=2, lens=[1], Q=strides(64, 64), Q_out=strides(64, 128)) == 1 and "same view" in error(mk)
    assert rotate(mk, desc(mk, q_per_kv=2, H=1), n=1, lens=[1], Q=strides(512, 64), Q_out=strides(4096, 64)) == 1 and "same view" in error(mk)


def views(mk, rng, B, base, sb, sh, st, lens):
    v = mk._CTensor(base, sb, sh, st, None)
    if rng.random() < 0.3:
        v.seq_start = (ct.c_int32 * B)(*[int(x) for x in rng.integers(0, 12, B)])
    return v


def test_an_output_that_overlaps_its_input(mk):
    """Random views of one buffer with the same strides, against the rows' bytes written out.  A call that is not refused fails to be launched here (there is no GPU)
    or has no rows."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the pointers are fake: calls that are taken would run")
    rng = np.random.default_rng(0)
    refused = taken = 0
    for _ in range(1500):
        B, H, g, n = (int(rng.integers(1, hi)) for hi in (4, 4, 3, 8))
        st = 64 * int(rng.integers(1, 5))
        sh = int(rng.choice([64, 64 * n, st * n, st * 9, 8 * int(rng.integers(0, 40))]))
        sb = int(rng.choice([sh * H * g, st * n, 64 * 100, 0]))
        lens = [int(x) for x in rng.integers(0, n + 1, B)]
        v, o = (views(mk, rng, B, 0x100000 + 16 * int(rng.integers(0, 1500)) * int(rng.random() < 0.8), sb, sh, st, lens) for _ in range(2))

        def rows(t):
            return {(t.ptr + 2 * (b * sb + h * sh + (i + (t.seq_start[b] if t.seq_start else 0)) * st)) // 16 + e
                    for b in range(B) for h in range(H * g) for i in range(lens[b]) for e in range(8)}

        start = lambda t: [t.ptr + 2 * (b * sb + (t.seq_start[b] if t.seq_start else 0) * st) for b in range(B)]
        meet = start(v) != start(o) and bool(rows(v) & rows(o))
        got = rotate(mk, desc(mk, B=B, H=H, q_per_kv=0 if g == 1 else g), n=n, lens=lens, Q=v, Q_out=o)
        assert (got == 1) == meet, (B, H, g, n, st, sh, sb, lens, got, error(mk))
        refused, taken = refused + meet, taken + (not meet)
    assert refused > 200 and taken > 200


def test_views_that_take_turns_in_one_buffer(mk):
    """Several views' heads of a token behind each other, and head by head in turn, as fused projections leave them: against the rows' bytes written out."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the pointers are fake: calls that are taken would run")
    rng = np.random.default_rng(1)
    refused = taken = 0
    for _ in range(1500):
        B, H, n, parts = (int(rng.integers(1, hi)) for hi in (4, 5, 8, 4))
        d = 64
        st = d * H * parts + int(rng.choice([0, 8, 64]))
        sh = d if rng.random() < 0.5 else d * parts
        sb = st * n * int(rng.integers(0, 2)) + 8 * int(rng.integers(0, 3))
        lens = [int(x) for x in rng.integers(0, n + 1, B)]
        at = lambda: 0x100000 + 2 * int(rng.choice([d, H * d, 8])) * int(rng.integers(0, 2 * parts + 1)) + 2 * st * int(rng.integers(0, 3))
        v, o = (views(mk, rng, B, at(), sb, sh, st, lens) for _ in range(2))

        def rows(t):
            return {(t.ptr + 2 * (b * sb + h * sh + (i + (t.seq_start[b] if t.seq_start else 0)) * st)) // 16 + e
                    for b in range(B) for h in range(H) for i in range(lens[b]) for e in range(8)}

        start = lambda t: [t.ptr + 2 * (b * sb + (t.seq_start[b] if t.seq_start else 0) * st) for b in range(B)]
        meet = start(v) != start(o) and bool(rows(v) & rows(o))
        got = rotate(mk, desc(mk, B=B, H=H), n=n, lens=lens, Q=v, Q_out=o)
        assert (got == 1) == meet, (B, H, n, parts, st, sh, sb, lens, got, error(mk))
        refused, taken = refused + meet, taken + (not meet)
    assert refused > 200 and taken > 200
