"""Attention over a cache in 4 bits against the float64 oracle over the values that the cache stands for."""
import numpy as np
import pytest
import torch

from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, B, H, d, dtype, n, lens, g=1, q_size=1.0, k_size=1.0, v_size=1.0):
        rng = np.random.default_rng(seed)
        self.B, self.H, self.d, self.dtype, self.n, self.g, self.lens = B, H, d, dtype, n, g, list(lens)
        total = sum(lens)
        self.Q = mh.gauss(rng, B, H * g, n, d, dtype=dtype, size=q_size)
        self.K, self.V = mh.gauss(rng, total, d, dtype=dtype, size=k_size), mh.gauss(rng, total, d, dtype=dtype, size=v_size)
        self.Kr, self.Vr = mh.gauss(rng, B, H, n, d, dtype=dtype, size=k_size), mh.gauss(rng, B, H, n, d, dtype=dtype, size=v_size)
        self.cu = mh.prefix(lens)
        self.P_max = max(list(lens) + [1])

    def run(self, capacity=None, scale=0.0, Q=None, Kr=None, Vr=None, O=None, with_lse=True, cache=None):
        m = hp.mk()
        capacity = int(self.cu[-1]) if capacity is None else capacity
        self.desc = mh.desc(self.B, self.H, self.d, self.dtype, self.n, self.P_max, self.g)
        cache = mh.cache(self.K, self.V, spare=max(capacity - int(self.cu[-1]), 0) + 3) if cache is None else cache
        up = lambda x: hp.upload(x, self.dtype)
        O = torch.full((self.B, self.H * self.g, self.n, self.d), 7.0, dtype=hp.torch_dtype(self.dtype), device="cuda") if O is None else O
        lse = torch.full((self.B * self.H * self.g * self.n,), 7.0, device="cuda") if with_lse else None
        ws = hp.workspace(m.maskkv_attend_mx_workspace_bytes(self.desc, capacity))
        m.maskkv_attend_mx(self.desc, up(self.Q) if Q is None else Q, cache, mh.device(self.cu), capacity, up(self.Kr) if Kr is None else Kr,
                           up(self.Vr) if Vr is None else Vr, scale, O, lse, ws)
        torch.cuda.synchronize()
        self.O = O.double().cpu().numpy()
        self.lse = None if lse is None else lse.double().cpu().numpy().reshape(self.B * self.H, self.g * self.n)
        return self

    def check(self, capacity=None, scale=None, heads=None):
        K, V = mh.stored(self.K), mh.stored(self.V)
        for i in range(self.B * self.H) if heads is None else heads:
            b, h = divmod(i, self.H)
            a, z = self.cu[i], self.cu[i + 1]
            if capacity is not None:
                a, z = min(a, capacity), min(z, capacity)
            rows = slice(h * self.g, (h + 1) * self.g)
            mh.check_attention(self.O[b, rows].reshape(-1, self.d), None if self.lse is None else self.lse[i],
                               self.Q[b, rows].reshape(-1, self.d), np.concatenate((K[a:z], self.Kr[b, h])),
                               np.concatenate((V[a:z], self.Vr[b, h])), self.dtype, scale, f"head {i}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 33, 64, 130])
def test_lengths_around_the_tiles(dtype, d, n):
    lens = [0, 1, 31, 32, 33, 63, 64, 65, 127, 129, 255, 300]
    Case(n + d, 2, 6, d, dtype, n, lens).run().check()


@pytest.mark.parametrize("dtype,g,n", [("bf16", 7, 1), ("bf16", 7, 5), ("bf16", 4, 40), ("bf16", 3, 129), ("f32", 7, 1), ("f32", 4, 9),
                                       ("bf16", 64, 3), ("bf16", 16, 1), ("bf16", 17, 1), ("bf16", 8, 2)])
def test_grouped_queries(dtype, g, n):
    Case(g + n, 2, 2, 128, dtype, n, [70, 0, 401, 33], g=g).run().check()
    Case(g + n, 1, 3, 64, dtype, n, [64, 1, 200], g=g).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 8, 40, 300])
def test_long_and_uneven_caches(dtype, n):
    """Few query rows over long caches: the key axis is dealt to several workgroups, and one head has nearly all the rows."""
    Case(n, 1, 2, 128, dtype, n, [5000, 3]).run().check()
    Case(n, 1, 3, 64, dtype, n, [0, 4097, 1500]).run().check()


def test_a_very_long_cache():
    Case(1, 1, 2, 128, "bf16", 1, [30011, 70000], g=7).run().check()


def test_many_heads_and_sequences():
    rng = np.random.default_rng(3)
    Case(3, 16, 20, 64, "bf16", 5, rng.integers(0, 90, 320).tolist()).run().check()
    Case(4, 64, 8, 64, "bf16", 1, rng.integers(0, 40, 512).tolist()).run().check()
    Case(5, 8, 32, 128, "bf16", 70, rng.integers(0, 300, 256).tolist()).run().check(heads=range(0, 256, 5))
    Case(6, 1, 600, 64, "bf16", 2, rng.integers(0, 30, 600).tolist()).run().check()


@pytest.mark.parametrize("n", [300, 512])
def test_more_queries_than_a_workgroup_has(n):
    Case(n, 2, 4, 128, "bf16", n, [100, 0, 513, 64, 1024, 31, 7, 200]).run().check()
    Case(n, 1, 2, 64, "bf16", n, [777, 3], g=4).run().check()


@pytest.mark.parametrize("d,n,g,lens", [(128, 300, 1, [24000, 100]), (64, 40, 7, [0, 30000]), (128, 70, 1, [9001, 40000, 17])])
def test_many_queries_over_few_long_heads(d, n, g, lens):
    """128 query rows a workgroup, and the keys of a head dealt to several."""
    Case(n, 1, len(lens), d, "bf16", n, lens, g=g).run().check()


@pytest.mark.parametrize("d,H,n", [(128, 16, 256), (64, 32, 384)])
def test_many_queries_over_long_heads(d, H, n):
    """128 query rows a workgroup, the keys of heads of several lengths dealt to several."""
    rng = np.random.default_rng(21)
    lens = rng.integers(3000, 5600, H)
    lens[[2, 5]] = [0, 9001]
    Case(21, 1, H, d, "bf16", n, lens.tolist()).run().check(heads=[0, 2, 5, H - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("BH,n", [(4, 478), (9, 100), (13, 33)])
def test_heads_that_the_xcds_do_not_share_evenly(dtype, BH, n):
    Case(22, 1, BH, 64, dtype, n, [11, 0, 40, 3, 90, 1, 64, 33, 17, 5, 32, 2, 100][:BH]).run().check()


def test_many_queries_of_many_heads():
    """128 query rows a workgroup, heads whole: in the order of their lengths, and more of them than are ordered."""
    rng = np.random.default_rng(18)
    Case(18, 1, 300, 64, "bf16", 70, rng.integers(0, 100, 300).tolist()).run().check(heads=range(0, 300, 7))
    lens = rng.integers(0, 200, 240)
    lens[[3, 77]] = 1500
    lens[100:110] = 0
    Case(19, 3, 80, 64, "bf16", 66, lens.tolist()).run().check(heads=[0, 3, 50, 77, 100, 105, 200, 239])


@pytest.mark.parametrize("n", [1, 20, 70])
def test_heads_that_may_be_long_where_the_launch_fills_the_chip(n):
    """Room for far longer heads than there are: the keys are dealt out all the same, and most heads have one part."""
    rng = np.random.default_rng(19)
    lens = rng.integers(0, 60, 260)
    lens[[5, 200]] = 2000
    c = Case(20, 2, 130, 64, "bf16", n, lens.tolist())
    c.P_max = 100000
    c.run(capacity=80000).check(heads=[0, 5, 6, 100, 200, 201, 259])


@pytest.mark.parametrize("capacity", [0, 1, 40, 99, 100, 101, 150])
def test_rows_are_clipped_to_the_capacity(capacity):
    c = Case(8, 1, 3, 64, "bf16", 9, [40, 0, 110])
    c.run(capacity=capacity).check(capacity=capacity)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 150])
def test_scale_and_large_logits(dtype, n):
    c = Case(9, 1, 2, 64, dtype, n, [200, 77], q_size=6.0, k_size=6.0, v_size=3.0)
    c.run(scale=0.7).check(scale=float(np.float32(0.7)))
    # every logit far below zero, and then far above: the running maximum starts from neither
    for sign in (-1.0, 1.0):
        c = Case(10, 1, 2, 64, dtype, n, [100, 0])
        c.Q[..., 0], c.K[:, 0], c.Kr[..., 0] = 40.0, sign * 48.0, sign * 48.0
        c.run().check()


def test_growing_logits_raise_the_reference_again_and_again():
    c = Case(11, 1, 1, 128, "bf16", 40, [900])
    c.Q[..., 5] = 3.0
    c.K[:, 5] = np.arange(900) // 16
    c.run().check()


@pytest.mark.parametrize("n", [1, 3, 100])
def test_other_orders_in_memory(n):
    c = Case(12, 2, 3, 128, "bf16", n, [20, 64, 1, 0, 90, 33], g=2)
    tokens = lambda x: hp.upload(x.transpose(0, 2, 1, 3).copy(), "bf16").transpose(1, 2)       # [B, T, H, d] in memory
    O = torch.full((2, n, 6, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    c.run(Q=tokens(c.Q), Kr=tokens(c.Kr), Vr=tokens(c.Vr), O=O.transpose(1, 2))
    c.check()
    # the response rows behind a prompt of each sequence's own length, O inside a wider tensor that keeps its other columns
    m = hp.mk()
    starts = [11, 4]
    full = np.zeros((2, 2, 3, 11 + n, 128), dtype=np.float32)
    for b in range(2):
        full[0, b, :, starts[b]:starts[b] + n], full[1, b, :, starts[b]:starts[b] + n] = c.Kr[b], c.Vr[b]
    wide = torch.full((2, 6, n, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    c.run(Kr=m.tensor_view(hp.upload(full[0], "bf16"), seq_start=starts), Vr=m.tensor_view(hp.upload(full[1], "bf16"), seq_start=starts),
          O=wide[..., 64:192], with_lse=False)
    c.check()
    assert (wide[..., :64] == 5.0).all() and (wide[..., 192:] == 5.0).all()


@pytest.mark.parametrize("n", [1, 40, 200])
def test_a_head_with_a_nan_is_nan_and_no_other(n):
    c = Case(13, 1, 3, 128, "bf16", n, [100, 100, 100])
    c.K[150, 7] = np.nan
    c.run().check(heads=(0, 2))
    assert np.isnan(c.O[0, 1]).all() and np.isnan(c.lse[1]).all()
    c = Case(14, 1, 3, 128, "bf16", n, [100, 100, 100])
    c.V[150, 40] = np.inf                                           # one group of the values' columns
    c.run().check(heads=(0, 2))
    assert np.isnan(c.O[0, 1, :, 32:64]).all() and np.isfinite(c.O[0, 1, :, :32]).all() and np.isfinite(c.lse).all()


def test_codes_behind_the_last_row_do_not_matter():
    """Rows past the end hold bytes that stand for NaN; so does what lies past a clipped head."""
    c = Case(15, 1, 2, 128, "bf16", 9, [33, 70])
    c.run(cache=mh.cache(c.K, c.V, spare=64, fill=0xFF)).check()


def test_the_same_call_gives_the_same_bits():
    for n, lens in ((1, [9000, 50]), (256, [300, 40])):
        c = Case(16, 1, 2, 128, "bf16", n, lens)
        first = c.run().O.copy()
        assert np.array_equal(first, c.run().O)


def test_agrees_with_the_attention_over_the_expanded_cache():
    m = hp.mk()
    c = Case(17, 2, 4, 128, "bf16", 100, [90, 20, 0, 300, 64, 1, 500, 33]).run()
    total = int(c.cu[-1])
    Kc, Vc = (torch.zeros(total, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m.maskkv_expand_mx(c.desc, mh.cache(c.K, c.V), mh.device(c.cu), total, Kc, Vc)
    O = torch.zeros(2, 4, 100, 128, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(800, device="cuda")
    up = lambda x: hp.upload(x, "bf16")
    m.maskkv_attend(c.desc, up(c.Q), Kc, Vc, mh.device(c.cu), total, up(c.Kr), up(c.Vr), 0.0, O, lse,
                    hp.workspace(m.maskkv_attend_workspace_bytes(c.desc, False)))
    O, lse = O.double().cpu().numpy(), lse.double().cpu().numpy().reshape(8, 100)
    for i in range(8):
        b, h = divmod(i, 4)
        a, z = c.cu[i], c.cu[i + 1]
        mh.check_attention(O[b, h], lse[i], c.Q[b, h], np.concatenate((mh.stored(c.K)[a:z], c.Kr[b, h])),
                           np.concatenate((mh.stored(c.V)[a:z], c.Vr[b, h])), "bf16")
    c.check()


def test_shapes_are_held_against_the_description():
    m = hp.mk()
    d = mh.desc(2, 2, 64, "bf16", 4, 10, g=2)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    Q, Kr, cu, cache = bf(2, 4, 4, 64), bf(2, 2, 4, 64), mh.device(mh.prefix([2, 3, 4, 1])), m.MxCache.empty(10, 64)
    lse = torch.zeros(32, device="cuda")
    good = [d, Q, cache, cu, 10, Kr, Kr.clone(), 0.0, Q.clone(), lse, None]
    m.maskkv_attend_mx(*good)
    torch.cuda.synchronize()
    for at, x in ((1, bf(2, 2, 4, 64)), (1, Q.float()), (3, cu[:4]), (3, cu.long()), (4, 11), (5, bf(2, 2, 3, 64)), (6, bf(1, 2, 4, 64)),
                  (8, bf(2, 4, 4, 128)), (9, lse[:31]), (9, lse.double()), (2, m.MxCache.empty(10, 64, device="cpu"))):
        with pytest.raises((AssertionError, TypeError)):
            m.maskkv_attend_mx(*(x if i == at else a for i, a in enumerate(good)))
