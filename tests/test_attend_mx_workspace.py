"""The workspace of maskkv_attend_mx: what is enough for a cache is enough for every smaller one (CPU)."""
import numpy as np
import pytest

SHAPES = [dict(B=1, H=4, d=128, n_resp=1, P_max=131072, q_per_kv=7), dict(B=1, H=32, d=128, n_resp=32, P_max=8192),
          dict(B=2, H=8, d=128, n_resp=256, P_max=16384, q_per_kv=4), dict(B=8, H=32, d=128, n_resp=512, P_max=32768),
          dict(B=1, H=2, d=64, n_resp=40, P_max=30000), dict(B=1, H=2, d=64, n_resp=40, P_max=30000, f32=True),
          dict(B=4, H=16, d=64, n_resp=100, P_max=65536, f32=True), dict(B=64, H=32, d=64, n_resp=4, P_max=4096)]


@pytest.fixture(scope="module")
def mk():
    from paper_2510_09309_amd import binding
    return binding


def description(mk, f32=False, **kw):
    return mk.Desc(dtype=mk.MASKKV_F32 if f32 else mk.MASKKV_BF16, **kw)


@pytest.mark.parametrize("kw", SHAPES)
def test_a_smaller_capacity_never_needs_more(mk, kw):
    d = description(mk, **kw)
    caps = sorted(set(range(0, 200)) | {int(c) for c in np.geomspace(200, 400000, 700)} | {2 ** k + e for k in range(8, 19) for e in (-1, 0, 1)})
    sizes = [mk.maskkv_attend_mx_workspace_bytes(d, c) for c in caps]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_what_shrinks_by_evictions(mk):
    """Capacities of caches that used to need more than the larger ones that they came from."""
    for kw, large, small in ((SHAPES[0], 131072, 91750), (SHAPES[1], 62259, 58982), (SHAPES[2], 95027, 85196)):
        d = description(mk, **kw)
        assert mk.maskkv_attend_mx_workspace_bytes(d, large) >= mk.maskkv_attend_mx_workspace_bytes(d, small) > 0


def test_the_largest_capacity_is_looked_over_too(mk):
    d = description(mk, **SHAPES[0])
    assert mk.maskkv_attend_mx_workspace_bytes(d, 0x7FFF0000) >= mk.maskkv_attend_mx_workspace_bytes(d, 131072)
