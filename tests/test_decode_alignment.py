"""maskkv_sample and maskkv_rotate refuse arrays of 32-bit entries that are not 4-byte aligned, before anything is enqueued (CPU: the pointers are fake)."""
import ctypes as ct

import pytest

from tests.test_decode_refusals import F, Sampling, error, mk, rotate  # noqa: F401  (mk: a fixture)


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("name", ["temperature", "top_k", "top_p", "min_p", "uniform", "token", "prob", "logprob"])
def test_sample(mk, name, off):
    given = dict(temperature=None, top_k=None, top_p=None, min_p=None, uniform=F, token=F, prob=None, logprob=None)
    given[name] = F + off
    s = Sampling(*(given[n] for n in ("temperature", "top_k", "top_p", "min_p", "uniform")))
    assert mk.raw_library().maskkv_sample(ct.c_void_p(F), ct.c_int64(2), ct.c_int32(100), ct.c_int32(1), ct.c_int64(100), ct.byref(s), ct.c_void_p(given["token"]),
                                          ct.c_void_p(given["prob"]), ct.c_void_p(given["logprob"]), ct.c_void_p(F), ct.c_size_t(1 << 20), None) == 1
    assert "aligned" in error(mk)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_rotate(mk, off):
    assert rotate(mk, positions=F + off) == 1 and "positions" in error(mk) and "aligned" in error(mk)
