"""What the calls of the 4-bit cache and of further eviction refuse, before anything is enqueued (CPU: the pointers are fake)."""
import ctypes as ct

import pytest
import torch

F = 0x10000


@pytest.fixture(scope="module")
def mk():
    from paper_2510_09309_amd import binding
    return binding


class Mx(ct.Structure):
    _fields_ = [(n, ct.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")]


class Calls:
    """The entry points with good (fake) arguments of one description; every keyword replaces one."""

    def __init__(self, mk, **kw):
        self.lib = mk.raw_library()
        self.desc = mk.Desc(**{**dict(B=1, H=2, d=64, dtype=mk.MASKKV_BF16, n_resp=8, P_max=100), **kw}).c()
        self.good = dict(view=mk._CTensor(F, 0, 108 * 64, 64, None), mx=Mx(F, F, F, F), out=Mx(*[F + (1 << 20) * i for i in (1, 2, 3, 4)]),
                         idx=F, cu=F, cap=10, cap_out=5, scale=0.0, lse=F, decay=0.5, w_in=F, w_out=F + (9 << 20), budgets=F, weights=F,
                         K=F, V=F, K_out=F + (1 << 20), V_out=F + (2 << 20), idx_out=F + (5 << 20), rows=F + (6 << 20),
                         cu_out=F + (7 << 20), ws=None, ws_bytes=0, O=F)

    def at(self, kw, name):
        v = {**self.good, **kw}[name]
        if isinstance(v, ct.Structure):
            return ct.byref(v)
        if name in ("cap", "cap_out"):
            return ct.c_int64(v)
        if name in ("scale", "decay"):
            return ct.c_float(v)
        return ct.c_size_t(v) if name == "ws_bytes" else ct.c_void_p(v)

    def call(self, what, names, kw):
        return getattr(self.lib, what)(ct.byref(self.desc), *(self.at(kw, n) for n in names.split()), None)

    def compact(self, **kw):
        return self.call("maskkv_compact_mx", "view view idx cu cap mx", kw)

    def expand(self, **kw):
        return self.call("maskkv_expand_mx", "mx cu cap K V", kw)

    def attend(self, **kw):
        o = {**kw}
        return self.call("maskkv_attend_mx", "view mx cu cap view view scale view lse ws ws_bytes", o)

    def accumulate(self, **kw):
        return self.call("maskkv_accumulate", "view K cu cap scale lse decay w_in w_out", kw)

    def accumulate_mx(self, **kw):
        return self.call("maskkv_accumulate_mx", "view mx cu cap scale lse decay w_in w_out", kw)

    def evict(self, **kw):
        return self.call("maskkv_evict", "weights cu cap budgets K V idx K_out V_out idx_out rows w_out cu_out cap_out", kw)

    def evict_mx(self, **kw):
        return self.call("maskkv_evict_mx", "weights cu cap budgets mx idx out idx_out rows w_out cu_out cap_out", kw)

    def error(self):
        return self.lib.maskkv_last_error().decode()


ALL = ("compact", "expand", "attend", "accumulate", "accumulate_mx", "evict", "evict_mx")


@pytest.mark.parametrize("what", ALL)
@pytest.mark.parametrize("kw,status", [(dict(d=96), 2), (dict(dtype=7), 3), (dict(B=0), 2), (dict(B=65), 2), (dict(n_resp=0), 1)])
def test_bad_descriptions(mk, what, kw, status):
    c = Calls(mk, **kw)
    assert getattr(c, what)() == status and c.error()


@pytest.mark.parametrize("what", ALL)
def test_bad_capacities_and_prefix_sums(mk, what):
    c = Calls(mk)
    assert getattr(c, what)(cap=-1) == 1 and "capacity" in c.error()
    assert getattr(c, what)(cap=1 << 31) == 1 and getattr(c, what)(cap=0x7FFF0001) == 1
    assert getattr(c, what)(cu=None) == 1 and "cu_budget" in c.error()


@pytest.mark.parametrize("what", ("compact", "expand", "attend", "accumulate_mx", "evict_mx"))
def test_bad_caches(mk, what):
    c = Calls(mk)
    assert getattr(c, what)(mx=None) == 1 and "cache" in c.error()
    for i, name in enumerate(("k_codes", "k_scales", "v_codes", "v_scales")):
        if what == "accumulate_mx" and i > 1:
            continue                                                           # the values are not looked at
        assert getattr(c, what)(mx=Mx(*(None if j == i else F for j in range(4)))) == 1 and name in c.error()
        assert getattr(c, what)(mx=Mx(*(F + 8 * (j == i) for j in range(4)))) == 1 and "aligned" in c.error()


@pytest.mark.parametrize("what", ("compact", "attend", "accumulate", "accumulate_mx"))
def test_bad_views(mk, what):
    c = Calls(mk)
    for view in (mk._CTensor(0, 0, 0, 64, None), mk._CTensor(F + 4, 0, 108 * 64, 64, None), mk._CTensor(F, 0, 108 * 64, 32, None),
                 mk._CTensor(F, 0, 0, (1 << 24) // 2 + 8, None)):
        assert getattr(c, what)(view=view) == 1


def test_bad_arguments_of_each_call(mk):
    c = Calls(mk)
    assert c.compact(idx=None) == 1 and "idx" in c.error()
    assert c.expand(K=None) == 1 and c.expand(V=F + 8) == 1 and "Vc" in c.error()
    for call in (c.accumulate, c.accumulate_mx):
        assert call(lse=None) == 1 and call(w_out=None) == 1 and call(w_in=None) == 1
        for decay in (-0.1, 1.5, float("nan")):
            assert call(decay=decay) == 1 and "decay" in c.error()
        for w_in in (F + (9 << 20) + 4, F + (9 << 20) - 36):                   # ten weights that overlap the other ten
            assert call(w_in=w_in) == 1 and "overlap" in c.error()
    assert c.accumulate(K=None) == 1 and "Kc" in c.error()
    for call in (c.evict, c.evict_mx):
        assert call(weights=None) == 1 and call(budgets=None) == 1 and call(cu_out=None) == 1 and call(rows=None) == 1
        assert call(idx=None) == 1 and call(idx_out=None) == 1 and "idx" in c.error()
        assert call(cap_out=-1) == 1 and "capacity_out" in c.error()
    assert c.evict(K_out=None) == 1 and c.evict(V=F + 2) == 1
    assert c.evict_mx(out=None) == 1 and c.evict_mx(out=Mx(F + (1 << 20), None, F, F)) == 1


def test_a_smaller_cache_that_overlaps_the_old_one_is_refused(mk):
    c = Calls(mk)
    rows = 10 * 128                                                            # bytes of Kc: 10 rows of 64 bf16
    for kw in (dict(K_out=F), dict(K_out=F + rows - 16), dict(V_out=F), dict(w_out=F), dict(cu_out=F), dict(rows=F), dict(idx_out=F + 16),
               dict(K_out=F + (2 << 20)), dict(rows=F + (7 << 20) + 4)):        # (the last two: two outputs)
        assert c.evict(**kw) == 1 and "overlaps" in c.error(), kw
    for i in range(4):
        out = Mx(*(F + 16 if j == i else F + (1 << 20) * (j + 1) for j in range(4)))
        assert c.evict_mx(out=out) == 1 and "overlaps" in c.error()


def test_heads_beyond_what_select_keeps_are_refused(mk):
    c = Calls(mk, P_max=(1 << 22) + 1)
    assert c.evict() == 2 and c.evict_mx() == 2 and "rows" in c.error()


def test_workspace_query(mk):
    d = mk.Desc(B=1, H=2, d=64, dtype=mk.MASKKV_BF16, n_resp=8, P_max=100)
    assert mk.maskkv_attend_mx_workspace_bytes(d, 0) >= 0
    with pytest.raises(mk.MaskKVError):
        mk.maskkv_attend_mx_workspace_bytes(d, -1)
    with pytest.raises(mk.MaskKVError):
        mk.maskkv_attend_mx_workspace_bytes(d, 1 << 31)
    with pytest.raises(mk.MaskKVError):
        mk.maskkv_attend_mx_workspace_bytes(mk.Desc(B=1, H=2, d=80, dtype=mk.MASKKV_BF16, n_resp=8, P_max=100), 10)


def test_the_binding_refuses_tensors_of_the_host(mk):
    d = mk.Desc(B=1, H=2, d=64, dtype=mk.MASKKV_BF16, n_resp=8, P_max=100)
    x, i, w = torch.zeros(1, 2, 108, 64).bfloat16(), torch.zeros(16, dtype=torch.int32), torch.zeros(16)
    rows = torch.zeros(10, 64).bfloat16()
    c = mk.MxCache.empty(10, 64, device="cpu")
    assert [t.shape for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales)] == [(10, 32), (10, 2)] * 2
    for call in (lambda: mk.maskkv_compact_mx(d, x, x, i, i, 10, c), lambda: mk.maskkv_expand_mx(d, c, i, 10, rows, rows),
                 lambda: mk.maskkv_attend_mx(d, x, c, i, 10, x, x, 0.0, x, w, None),
                 lambda: mk.maskkv_accumulate(d, x, rows, i, 10, 0.0, w, 0.0, None, w),
                 lambda: mk.maskkv_accumulate_mx(d, x, c, i, 10, 0.0, w, 0.0, None, w),
                 lambda: mk.maskkv_evict(d, w, i, 10, i, rows, rows, None, rows, rows, None, i, w, i, 5),
                 lambda: mk.maskkv_evict_mx(d, w, i, 10, i, c, None, c, None, i, w, i, 5)):
        with pytest.raises((AssertionError, TypeError)):
            call()
