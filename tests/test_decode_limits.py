"""Launches that would have 2^32 threads or more are refused, as the header says, before anything is enqueued (CPU: the pointers are fake)."""
import ctypes as ct

import pytest

from tests.test_decode_refusals import F, Sampling, attend, desc, error, mk  # noqa: F401  (mk: a fixture)


@pytest.mark.parametrize("dtype", [0, 1])
def test_attend_tree(mk, dtype):
    """B * H * query rows beyond 2^27 may be more than a launch can have; 2^33 is."""
    d = desc(mk, B=64, H=1000, n_resp=1 << 17, P_max=0, dtype=dtype)
    n = ct.c_size_t(0)
    assert mk.raw_library().maskkv_attend_tree_workspace_bytes(ct.byref(d), ct.c_int64(0), ct.byref(n)) == 0
    assert attend(mk, d, cap=0, K=None, V=None, ws=F, ws_bytes=1 << 60) == 2 and "launch" in error(mk)


def test_all_that_the_header_promises_can_be_launched(mk):
    """2^27 query rows of any shape, and any cache: the plan's workgroups have fewer than 2^32 threads."""
    import numpy as np
    from paper_2510_09309_amd import bench_binding as bb
    rng = np.random.default_rng(0)
    for _ in range(3000):
        heads = int(np.exp(rng.uniform(0, np.log(65000))))
        n_resp = max(1, min((1 << 27) // heads, 1 << 20) - int(rng.integers(0, 3)))
        d = mk.Desc(B=1, H=heads, d=int(rng.choice([64, 128])), dtype=int(rng.integers(0, 2)), n_resp=n_resp, P_max=int(np.exp(rng.uniform(0, 16))))
        p = bb.maskkv_bench_attend_tree_plan(d, int(np.exp(rng.uniform(0, 21))))
        assert p.units * p.qtiles * 512 < 1 << 32


def test_sample(mk):
    s = Sampling(None, None, None, None, F)

    def call(rows, vocab, dtype):
        return mk.raw_library().maskkv_sample(ct.c_void_p(F), ct.c_int64(rows), ct.c_int32(vocab), ct.c_int32(dtype), ct.c_int64(vocab), ct.byref(s), ct.c_void_p(F),
                                              None, None, ct.c_void_p(F), ct.c_size_t(1 << 62), None)

    assert call(1 << 20, 1 << 24, 1) == 2 and "launch" in error(mk)
    assert call(1 << 20, 1 << 17, 0) == 2                         # 128 parts of 4 KB a row, and one for rows that begin anywhere
    assert call(1 << 20, 1 << 18, 1) == 2
