"""What maskkv_rotate, maskkv_tree_mask, maskkv_attend_tree and maskkv_sample refuse, before anything is enqueued (CPU: the pointers are fake)."""
import ctypes as ct
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as do

F = 0x10000


@pytest.fixture(scope="module")
def mk():
    from paper_2510_09309_amd import binding
    return binding


def error(mk):
    return mk.raw_library().maskkv_last_error().decode()


def desc(mk, **kw):
    return mk.Desc(**{**dict(B=1, H=2, d=64, dtype=mk.MASKKV_BF16, n_resp=8, P_max=1000), **kw}).c()


def view(mk, ptr=F, **kw):
    v = dict(b=0, h=108 * 64, t=64, start=None, **kw)
    return mk._CTensor(ptr, v["b"], v["h"], v["t"], v["start"])


def rotate(mk, d=None, rotary="good", positions=F, n=8, lens=None, Q="good", Q_out="good", K=None, K_out=None):
    r = mk.maskkv_rotary_frequencies(64) if rotary == "good" else rotary
    q = view(mk) if Q == "good" else Q
    o = view(mk, F << 8) if Q_out == "good" else Q_out
    ref = lambda x: None if x is None else ct.byref(x)
    arr = None if lens is None else (ct.c_int32 * len(lens))(*lens)
    return mk.raw_library().maskkv_rotate(ref(d or desc(mk)), ref(r), ct.c_void_p(positions), ct.c_int32(n), arr, ref(q), ref(o), ref(K), ref(K_out), None)


@pytest.mark.parametrize("kw,status", [(dict(d=96), 2), (dict(dtype=7), 3), (dict(B=0), 2), (dict(B=65), 2), (dict(q_per_kv=65), 1)])
def test_bad_descriptions(mk, kw, status):
    assert rotate(mk, desc(mk, **kw)) == status and attend(mk, desc(mk, **kw)) == status


def test_rotate_refuses(mk):
    assert rotate(mk, rotary=None) == 1 and "rotary" in error(mk)
    for width in (0, -2, 3, 66, 128):
        assert rotate(mk, rotary=mk.Rotary(width=width, layout=0, amplitude=1.0)) == 1 and "width" in error(mk)
    assert rotate(mk, rotary=mk.Rotary(width=64, layout=2, amplitude=1.0)) == 1 and "layout" in error(mk)
    bad = mk.maskkv_rotary_frequencies(64)
    bad.freq[31] = math.nan
    assert rotate(mk, rotary=bad) == 1 and "finite" in error(mk)
    for amplitude in (math.inf, math.nan, 1e39):                                 # (the last: beyond 32 bits)
        assert rotate(mk, rotary=mk.Rotary(width=64, layout=0, amplitude=amplitude)) == 1 and "finite" in error(mk)
    assert rotate(mk, positions=None) == 1 and "positions" in error(mk)
    assert rotate(mk, n=-1) == 1 and rotate(mk, n=(1 << 25) + 1) == 1 and "n_tokens" in error(mk)
    assert rotate(mk, lens=[9]) == 1 and rotate(mk, lens=[-1]) == 1 and "token_len" in error(mk)
    assert rotate(mk, Q=None) == 1 and rotate(mk, Q_out=None) == 1 and "Q" in error(mk)
    assert rotate(mk, Q=None, Q_out=None) == 1 and "neither" in error(mk)
    assert rotate(mk, K=view(mk)) == 1 and rotate(mk, K_out=view(mk)) == 1 and "K" in error(mk)
    assert rotate(mk, Q=view(mk, F + 4)) == 1 and rotate(mk, Q_out=view(mk, 0)) == 1
    other = view(mk)
    other.stride_t = 128
    assert rotate(mk, Q_out=other) == 1 and "same view" in error(mk)            # begins where Q does, and is another view
    assert rotate(mk, n=0, positions=None) == 0                                  # nothing to do
    assert rotate(mk, n=4, lens=[0]) == 0


def test_frequencies(mk):
    names = {"plain": mk.ROTARY_PLAIN, "linear": mk.ROTARY_LINEAR, "base": mk.ROTARY_BASE, "bands": mk.ROTARY_BANDS}
    for width in (2, 6, 64, 128):
        for name, scaling in names.items():
            for factor in (1.0, 4.0, 13.5):
                r = mk.maskkv_rotary_frequencies(width, mk.ROTARY_PAIRS, 500000.0, scaling, factor, 8192.0, 1.0, 32.0)
                want, amplitude = do.frequencies(width, 500000.0, name, factor, 8192.0, 1.0, 32.0)
                assert (r.width, r.layout) == (width, mk.ROTARY_PAIRS)
                # (a power, a product and a quotient: a few roundings each)
                assert np.allclose(r.freq[:width // 2], want, rtol=1e-14, atol=0) and r.amplitude == pytest.approx(amplitude, rel=1e-15)
                assert all(f == 0.0 for f in r.freq[width // 2:])
    for args in ((0,), (130,), (63,), (64, 2), (64, 0, 0.0), (64, 0, -1.0), (64, 0, math.inf), (64, 0, math.nan), (64, 0, 1e4, 4), (64, 0, 1e4, 1, 0.5),
                 (64, 0, 1e4, 1, math.inf), (64, 0, 1e4, 3, 2.0, 0.0), (64, 0, 1e4, 3, 2.0, 100.0, 3.0, 3.0), (64, 0, 1e4, 3, 2.0, 100.0, -1.0, 3.0)):
        with pytest.raises(mk.MaskKVError) as e:
            mk.maskkv_rotary_frequencies(*args)
        assert e.value.status == 1
    assert mk.raw_library().maskkv_rotary_frequencies(ct.c_int32(64), ct.c_int32(0), ct.c_double(1e4), ct.c_int32(0), ct.c_double(1), ct.c_double(0),
                                                      ct.c_double(0), ct.c_double(0), None) == 1


def attend(mk, d=None, **kw):
    g = {**dict(Q=view(mk), K=F, V=F, cu=F, cap=10, Kr=view(mk), Vr=view(mk), mask=F, O=view(mk), ws=None, ws_bytes=0), **kw}
    ref = lambda x: None if x is None else ct.byref(x)
    return mk.raw_library().maskkv_attend_tree(ref(d or desc(mk)), ref(g["Q"]), ct.c_void_p(g["K"]), ct.c_void_p(g["V"]), ct.c_void_p(g["cu"]),
                                               ct.c_int64(g["cap"]), ref(g["Kr"]), ref(g["Vr"]), ct.c_void_p(g["mask"]), ct.c_float(0.0), ref(g["O"]),
                                               None, ct.c_void_p(g["ws"]), ct.c_size_t(g["ws_bytes"]), None)


def test_attend_tree_refuses(mk):
    for name in ("Q", "Kr", "Vr", "O"):
        assert attend(mk, **{name: None}) == 1 and attend(mk, **{name: view(mk, F + 8)}) == 1
    for name in ("mask", "cu"):
        assert attend(mk, **{name: None}) == 1 and "NULL" in error(mk)
        assert attend(mk, **{name: F + 2}) == 1 and "aligned" in error(mk)
    assert attend(mk, K=None) == 1 and attend(mk, V=F + 8) == 1 and "Vc" in error(mk)
    for cap in (-1, 1 << 31, 0x7FFF0001):
        assert attend(mk, cap=cap) == 1 and "capacity" in error(mk)
    d = desc(mk, P_max=20000, n_resp=1)
    n = ct.c_size_t(0)
    assert mk.raw_library().maskkv_attend_tree_workspace_bytes(ct.byref(d), ct.c_int64(40000), ct.byref(n)) == 0 and n.value > 0
    assert attend(mk, d, cap=40000) == 4 and attend(mk, d, cap=40000, ws=F, ws_bytes=1000) == 4
    assert attend(mk, d, cap=40000, ws=F + 128, ws_bytes=n.value) == 4 and "aligned" in error(mk)
    assert mk.raw_library().maskkv_attend_tree_workspace_bytes(ct.byref(d), ct.c_int64(40000), None) == 1
    assert mk.raw_library().maskkv_attend_tree_workspace_bytes(ct.byref(d), ct.c_int64(-1), ct.byref(n)) == 1


def test_a_workspace_is_enough_for_every_smaller_cache(mk):
    """A program that goes on evicting keeps the workspace of its first cache; a call with less than the query says is only made with what
    the launch itself needs."""
    rng = np.random.default_rng(0)
    for _ in range(300):
        d = mk.Desc(B=int(rng.integers(1, 9)), H=int(rng.integers(1, 65)), d=int(rng.choice([64, 128])), dtype=int(rng.integers(0, 2)),
                    n_resp=int(np.exp(rng.uniform(0, 7))), P_max=int(np.exp(rng.uniform(0, 12))), q_per_kv=int(rng.choice([0, 2, 7])))
        sizes = [mk.maskkv_attend_tree_workspace_bytes(d, int(c)) for c in sorted(np.exp(rng.uniform(0, 15, 12)).astype(int))]
        assert sizes == sorted(sizes)


def test_tree_mask_refuses(mk):
    lib = mk.raw_library()
    call = lambda p, B, n, m: lib.maskkv_tree_mask(ct.c_void_p(p), ct.c_int32(B), ct.c_int32(n), ct.c_void_p(m), None)
    assert call(F, -1, 4, F) == 2 and call(F, 65536, 4, F) == 2 and call(F, 1, -1, F) == 2 and call(F, 1, (1 << 20) + 1, F) == 2
    assert call(None, 1, 4, F) == 1 and call(F, 1, 4, None) == 1 and call(F + 2, 1, 4, F) == 1 and call(F, 1, 4, F + 1) == 1
    assert call(None, 0, 4, None) == 0 and call(None, 3, 0, None) == 0


class Sampling(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p", "uniform")]


def sample(mk, logits=F, rows=2, vocab=100, dtype=1, stride=100, sampling="good", token=F, ws=F, ws_bytes=1 << 20):
    s = Sampling(None, None, None, None, F) if sampling == "good" else sampling
    return mk.raw_library().maskkv_sample(ct.c_void_p(logits), ct.c_int64(rows), ct.c_int32(vocab), ct.c_int32(dtype), ct.c_int64(stride),
                                          None if s is None else ct.byref(s), ct.c_void_p(token), None, None, ct.c_void_p(ws), ct.c_size_t(ws_bytes), None)


def test_sample_refuses(mk):
    assert sample(mk, dtype=2) == 3
    for kw in (dict(rows=-1), dict(rows=(1 << 20) + 1), dict(vocab=0), dict(vocab=-5), dict(vocab=(1 << 24) + 1, stride=1 << 25)):
        assert sample(mk, **kw) == 2 and "sample" in error(mk)
    assert sample(mk, stride=99) == 1 and sample(mk, stride=1 << 62) == 1 and sample(mk, sampling=None) == 1
    assert sample(mk, logits=None) == 1 and sample(mk, token=None) == 1 and sample(mk, sampling=Sampling()) == 1
    assert sample(mk, logits=F + 1) == 1 and sample(mk, logits=F + 2, dtype=0) == 1 and "aligned" in error(mk)
    assert sample(mk, ws=None) == 4 and sample(mk, ws_bytes=100) == 4 and sample(mk, ws=F + 16) == 4
    assert sample(mk, rows=0, logits=None, token=None, ws=None, ws_bytes=0) == 0
    n = ct.c_size_t(0)
    lib = mk.raw_library()
    query = lambda r, v, t, p=None: lib.maskkv_sample_workspace_bytes(ct.c_int64(r), ct.c_int32(v), ct.c_int32(t), p)
    assert query(1, 100, 1) == 1 and query(1, 0, 1, ct.byref(n)) == 2 and query(1, 100, 9, ct.byref(n)) == 3
    assert [mk.maskkv_sample_workspace_bytes(r, 32001, 1) for r in (0, 1, 2, 300)] == sorted(mk.maskkv_sample_workspace_bytes(r, 32001, 1)
                                                                                           for r in (0, 1, 2, 300))


def test_the_binding_refuses_tensors_of_the_host(mk):
    d = mk.Desc(B=1, H=2, d=64, dtype=mk.MASKKV_BF16, n_resp=8, P_max=100)
    x, i, w = torch.zeros(1, 2, 108, 64).bfloat16(), torch.zeros(16, dtype=torch.int32), torch.zeros(16)
    rows, r = torch.zeros(10, 64).bfloat16(), mk.maskkv_rotary_frequencies(64)
    for call in (lambda: mk.maskkv_rotate(d, r, i, 8, x, x, None, None), lambda: mk.maskkv_rotate(d, None, i, 8, x, x, None, None),
                 lambda: mk.maskkv_rotate(d, r, i, 1 << 40, x, x, None, None),
                 lambda: mk.maskkv_attend_tree(d, x, rows, rows, i, 10, x, x, i, 0.0, x, w, None),
                 lambda: mk.maskkv_tree_mask(i.view(2, 8), i), lambda: mk.maskkv_tree_mask(i, i),
                 lambda: mk.maskkv_sample(torch.zeros(2, 8), None, None, None, None, w, i, None, None, None),
                 lambda: mk.maskkv_sample(torch.zeros(2, 2, 8), None, None, None, None, w, i, None, None, None)):
        with pytest.raises((AssertionError, TypeError, ValueError)):
            call()
