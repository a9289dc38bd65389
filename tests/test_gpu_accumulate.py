"""The attention that cached rows get, added up, against the float64 oracle: caches of rows and in 4 bits."""
import numpy as np
import pytest
import torch

from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu


def check(seed, B, H, d, dtype, n, lens, mx, g=1, decay=0.0, capacity=None, scale=0.0, edit=None, in_place=False, heads=None, q_size=1.0,
          order=False):
    m = hp.mk()
    rng = np.random.default_rng(seed)
    total = sum(lens)
    cu = mh.prefix(lens)
    Q, K = mh.gauss(rng, B, H * g, n, d, dtype=dtype, size=q_size), mh.gauss(rng, total, d, dtype=dtype)
    # normalisers as an attention over these and other keys would return them: a little above the rows' own
    lse = (3.0 + rng.random((B * H, g * n)) + 0.5 * q_size ** 2 + np.log(np.maximum(lens, 1))[:, None]).astype(np.float32)
    before = rng.random(total + 5).astype(np.float32) * 3
    if edit:
        edit(Q, K, lse)
    capacity = total if capacity is None else capacity
    desc = mh.desc(B, H, d, dtype, n, max(list(lens) + [1]), g)
    out = torch.full((max(capacity, total) + 5,), 7.0, device="cuda")
    inp = mh.device(np.concatenate((before, np.zeros(max(capacity - total, 0), np.float32))))
    if in_place:
        out = inp
    Qd = hp.upload(Q.transpose(0, 2, 1, 3).copy(), dtype).transpose(1, 2) if order else hp.upload(Q, dtype)
    args = (mh.device(cu), capacity, scale, mh.device(lse.ravel()), decay, inp if decay else None, out)
    pad = np.zeros((max(capacity - total, 0), d), np.float32)
    if mx:
        c = mh.cache(K, K, spare=max(capacity - total, 0), fill=0xFF)
        m.maskkv_accumulate_mx(desc, Qd, m.MxCache(c.k_codes, c.k_scales), *args)
        K = mh.stored(K)
    else:
        m.maskkv_accumulate(desc, Qd, hp.upload(np.concatenate((K, pad + np.nan)), dtype), *args)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    assert np.array_equal(got[min(total, capacity):], inp.double().cpu().numpy()[min(total, capacity):] if in_place
                          else np.full(got.size - min(total, capacity), 7.0))
    for i in range(B * H) if heads is None else heads:
        b, h = divmod(i, H)
        a, z = min(cu[i], capacity), min(cu[i + 1], capacity)
        mh.check_weights(got[a:z], Q[b, h * g:(h + 1) * g].reshape(-1, d), K[a:z], lse[i].astype(np.float64), np.float64(np.float32(decay)),
                         before[a:z].astype(np.float64), None if scale == 0.0 else float(np.float32(scale)), f"head {i}")
    return got


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 15, 32, 33, 100, 257])
def test_lengths_around_the_tiles(mx, dtype, d, n):
    check(n + d, 2, 5, d, dtype, n, [0, 1, 31, 32, 33, 64, 100, 127, 129, 300], mx, decay=0.5)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("dtype,g,n", [("bf16", 7, 1), ("bf16", 7, 33), ("bf16", 64, 2), ("f32", 4, 10), ("bf16", 3, 200)])
def test_grouped_queries_add_up(mx, dtype, g, n):
    check(g + n, 2, 2, 128, dtype, n, [70, 0, 401, 33], mx, g=g)


@pytest.mark.parametrize("mx", [False, True])
def test_long_and_many(mx):
    check(1, 1, 2, 128, "bf16", 1, [30011, 2], mx)
    check(2, 1, 3, 64, "bf16", 40, [5, 4097, 900], mx, decay=1.0)
    rng = np.random.default_rng(3)
    check(3, 16, 20, 64, "bf16", 6, rng.integers(0, 50, 320).tolist(), mx)
    check(4, 1, 600, 64, "bf16", 2, rng.integers(0, 20, 600).tolist(), mx)
    check(5, 4, 8, 128, "bf16", 512, rng.integers(64, 700, 32).tolist(), mx, heads=(0, 7, 19, 31))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("d,dtype,n,g", [(64, "bf16", 300, 1), (128, "bf16", 130, 1), (64, "f32", 70, 1), (64, "bf16", 50, 3), (128, "bf16", 33, 2)])
def test_many_rows_share_the_queries(mx, d, dtype, n, g):
    """So many cached rows that a workgroup's waves share the queries: one step of 32 to ten, whole ones and a rest."""
    rng = np.random.default_rng(n)
    check(n, 8, 32, d, dtype, n, rng.integers(60, 260, 256).tolist(), mx, g=g, decay=0.5, heads=(0, 1, 99, 200, 255))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("capacity", [0, 1, 50, 59, 60, 61, 100])
def test_rows_are_clipped_to_the_capacity(mx, capacity):
    check(6, 1, 3, 64, "bf16", 9, [40, 0, 20], mx, decay=0.25, capacity=capacity)


@pytest.mark.parametrize("mx", [False, True])
def test_in_place_scale_and_order(mx):
    check(7, 1, 2, 128, "bf16", 20, [90, 33], mx, decay=0.9, in_place=True)
    check(8, 2, 2, 64, "f32", 20, [90, 33, 1, 0], mx, decay=1.0, in_place=True, scale=0.3)
    check(9, 2, 3, 128, "bf16", 33, [90, 33, 1, 0, 5, 64], mx, order=True, g=2)
    check(10, 1, 2, 64, "bf16", 40, [90, 33], mx, q_size=5.0)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("n", [3, 40, 200])
def test_rows_without_a_weight(mx, n):
    """A query row whose normaliser is +infinity adds nothing, and neither do all of them."""
    def some(Q, K, lse):
        lse[:, ::2] = np.inf
    check(11, 1, 2, 64, "bf16", n, [50, 40], mx, edit=some)

    def not_even_numbers(Q, K, lse):
        lse[:, 1::2], Q[:, :, 1::2] = np.inf, np.nan
    check(15, 1, 2, 64, "bf16", n, [50, 40], mx, edit=not_even_numbers)
    check(16, 1, 2, 128, "f32", n, [50, 40], mx, edit=not_even_numbers)

    def all_of_them(Q, K, lse):
        lse[:] = np.inf
    got = check(12, 1, 2, 64, "bf16", n, [50, 40], mx, edit=all_of_them)
    assert (got[:90] == 0.0).all()


def test_decay_of_nothing_reads_nothing():
    """With decay 0 the old weights do not count, not even as NaN."""
    m = hp.mk()
    rng = np.random.default_rng(13)
    Q, K = hp.upload(mh.gauss(rng, 1, 1, 8, 64), "bf16"), hp.upload(mh.gauss(rng, 30, 64), "bf16")
    desc, cu, lse = mh.desc(1, 1, 64, "bf16", 8, 30), mh.device(mh.prefix([30])), torch.full((8,), 4.0, device="cuda")
    a, b = torch.full((30,), float("nan"), device="cuda"), torch.zeros(30, device="cuda")
    m.maskkv_accumulate(desc, Q, K, cu, 30, 0.0, lse, 0.0, a, a)
    m.maskkv_accumulate(desc, Q, K, cu, 30, 0.0, lse, 0.0, None, b)
    assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("mx", [False, True])
def test_the_same_call_gives_the_same_bits(mx):
    for n, lens in ((1, [9000, 50]), (256, [300, 40])):
        a, b = (check(14, 1, 2, 128, "bf16", n, lens, mx, decay=0.5) for _ in range(2))
        assert np.array_equal(a, b)


def test_shapes_are_held_against_the_description():
    m = hp.mk()
    d = mh.desc(1, 2, 64, "bf16", 4, 10, g=2)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    f = lambda k: torch.zeros(k, device="cuda")
    good = [d, bf(1, 4, 4, 64), bf(10, 64), mh.device(mh.prefix([2, 3])), 10, 0.0, f(16), 0.5, f(10), f(10)]
    m.maskkv_accumulate(*good)
    torch.cuda.synchronize()
    for at, x in ((1, bf(1, 2, 4, 64)), (2, bf(9, 64)), (2, f(640)), (3, good[3][:2]), (6, f(15)), (8, f(9)), (9, f(9)), (9, f(10).double()),
                  (9, f(20)[::2])):
        with pytest.raises((AssertionError, TypeError)):
            m.maskkv_accumulate(*(x if i == at else a for i, a in enumerate(good)))
    with pytest.raises(m.MaskKVError):
        m.maskkv_accumulate(*(None if i == 8 else a for i, a in enumerate(good)))
