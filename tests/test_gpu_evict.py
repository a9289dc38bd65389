"""Further eviction from a packed cache against the oracle: which rows stay, and that whole rows move."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mxo
from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu


def check(lens, budgets, weights, d=64, dtype="bf16", mx=False, B=1, capacity=None, capacity_out=None, with_idx=True, with_weights=True):
    """Rows of random bytes: every one that stays has to arrive whole, and nothing else may be written."""
    m = hp.mk()
    rng = np.random.default_rng(len(lens) + sum(lens))
    lens, BH, total = list(lens), len(lens), sum(lens)
    cu = mh.prefix(lens)
    capacity = total if capacity is None else capacity
    bounds = [(min(cu[i], capacity), min(cu[i + 1], capacity)) for i in range(BH)]
    keep = [a + mxo.stay(weights[a:z], budgets[i]) for i, (a, z) in enumerate(bounds)]
    cu_want = mh.prefix([len(k) for k in keep])
    rows_want = np.concatenate(keep + [np.zeros(0, int)]).astype(np.int32)
    capacity_out = int(cu_want[-1]) if capacity_out is None else capacity_out
    written = min(int(cu_want[-1]), capacity_out)
    desc = mh.desc(B, BH // B, d, dtype, 1, max(lens + [1]))
    widths = [d // 2, d // 32, d // 2, d // 32] if mx else [d * (2 if dtype == "bf16" else 4)] * 2
    have = max(capacity, total)
    src = [rng.integers(0, 256, (have, w)).astype(np.uint8) for w in widths]
    dst = [torch.full((capacity_out + 4, w), 0x5A, dtype=torch.uint8, device="cuda") for w in widths]
    typed = lambda t: t if mx else t.view(hp.torch_dtype(dtype))
    dev = [typed(mh.device(x)) for x in src]
    out = [typed(t) for t in dst]
    idx = mh.device(rng.integers(0, 1 << 30, have).astype(np.int32)) if with_idx else None
    fill = lambda t, k=capacity_out: torch.full((k + 4,), 7, dtype=t, device="cuda")
    idx_out, rows, w_out = fill(torch.int32) if with_idx else None, fill(torch.int32), fill(torch.float32) if with_weights else None
    cu_out = torch.full((BH + 1,), -1, dtype=torch.int32, device="cuda")
    wd = mh.device(np.concatenate((weights, np.zeros(have - total, np.float32))).astype(np.float32))
    head = (desc, wd, mh.device(cu), capacity, mh.device(np.asarray(budgets, dtype=np.int32)))
    tail = (idx_out, rows, w_out, cu_out, capacity_out)
    if mx:
        m.maskkv_evict_mx(*head, m.MxCache(*dev), idx, m.MxCache(*out), *tail)
    else:
        m.maskkv_evict(*head, *dev, idx, *out, *tail)
    torch.cuda.synchronize()
    assert np.array_equal(cu_out.cpu().numpy(), cu_want)
    got = rows.cpu().numpy()
    assert np.array_equal(got[:written], rows_want[:written]) and (got[written:] == 7).all()
    for x, t in zip(src, dst):
        y = t.cpu().numpy()
        assert np.array_equal(y[:written], x[rows_want[:written]]) and (y[written:] == 0x5A).all()
    pairs = ([(idx, idx_out)] if with_idx else []) + ([(wd, w_out)] if with_weights else [])
    for x, t in pairs:
        x, y = x.cpu().numpy().view(np.int32), t.cpu().numpy()
        assert np.array_equal(y[:written].view(np.int32), x[rows_want[:written]]) and (y[written:] == 7).all()


def heavy(rng, n):
    return np.exp(2 * rng.standard_normal(n)).astype(np.float32)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32")])
def test_lengths_and_budgets(mx, d, dtype):
    rng = np.random.default_rng(d)
    lens = [0, 1, 2, 31, 63, 64, 65, 100, 255, 256, 257, 500, 1000, 0, 1023, 1024, 1025, 1, 64, 700]
    budgets = [5, 0, 1, 31, 30, 64, 1, 200, 128, 100, 256, 1, 999, 0, 512, 1024, 1000, 1, -3, 350]
    check(lens, budgets, heavy(rng, sum(lens)), d, dtype, mx, B=2)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("n,k", [(2048, 1000), (2049, 2048), (4096, 1), (4097, 3000), (8191, 5000), (16384, 16000), (16385, 7), (33000, 12345),
                                 (70000, 4096)])
def test_long_heads(mx, n, k):
    rng = np.random.default_rng(n)
    check([30, n, 7], [10, k, 7], heavy(rng, n + 37), 128, "bf16", mx)


@pytest.mark.parametrize("mx", [False, True])
def test_heads_of_all_lengths_listed_by_a_launch_of_their_own(mx):
    rng = np.random.default_rng(8)
    lens = [2049, 5000, 2048, 1, 4096, 3001, 0, 33000, 100, 12000]
    check(lens, [1000, 4999, 2047, 1, 1, 3001, 5, 20000, 99, 64], heavy(rng, sum(lens)), 64, "bf16", mx, B=2)


def test_a_long_head_among_short_ones():
    rng = np.random.default_rng(6)
    for n in (700, 3000, 4097, 9000):
        lens = [10] * 120 + [n] + [5] * 80
        check(lens, [4] * 120 + [n // 3] + [5] * 80, heavy(rng, sum(lens)), mx=n == 3000)


def test_ties():
    rng = np.random.default_rng(1)
    for n in (5, 64, 300, 1500, 5000, 20000):
        w = rng.integers(0, 4, n).astype(np.float32)                  # a few values only
        for k in (0, 1, n // 7, n // 2, n - 1, n):
            check([n], [k], w, mx=True)
        check([n, n], [n // 3, n // 2], np.zeros(2 * n, np.float32))  # nothing but ties


def test_weights_that_are_no_ordinary_numbers():
    rng = np.random.default_rng(2)
    special = np.array([0.0, -0.0, np.nan, -np.nan, np.inf, -np.inf, 1e-45, -1e-45, 3.4e38, -3.4e38, 1.0, -1.0], dtype=np.float32)
    for n in (12, 100, 3000):
        w = np.concatenate((special, special[rng.integers(0, 12, n - 12)]))
        for k in (1, 2, 5, n // 2, n - 1):
            check([n], [k], w)
    check([6], [4], np.full(6, np.nan, np.float32))
    check([6], [4], -np.arange(6, dtype=np.float32))
    # weights that differ in their last bit only
    w = (np.float32(1.0).view(np.int32) + rng.permutation(2000).astype(np.int32)).view(np.float32)
    check([2000], [777], w)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("capacity,capacity_out", [(100, None), (90, None), (35, None), (0, 0), (120, 70), (100, 30), (100, 0), (100, 200),
                                                   (None, 41)])
def test_capacities(mx, capacity, capacity_out):
    rng = np.random.default_rng(3)
    check([40, 0, 60], [30, 9, 20], heavy(rng, 100), mx=mx, capacity=capacity, capacity_out=capacity_out)


def test_without_positions_or_weights():
    rng = np.random.default_rng(4)
    check([40, 60], [30, 20], heavy(rng, 100), with_idx=False)
    check([40, 60], [30, 20], heavy(rng, 100), mx=True, with_weights=False)
    check([40, 60], [30, 20], heavy(rng, 100), with_idx=False, with_weights=False)


def test_many_heads():
    rng = np.random.default_rng(5)
    for BH, B in ((256, 8), (1024, 64), (3000, 1)):
        lens = rng.integers(0, 60, BH)
        check(lens.tolist(), rng.integers(0, 50, BH).tolist(), heavy(rng, int(lens.sum())), B=B, mx=BH == 1024)


def test_rows_beyond_four_gibibytes():
    """70 million rows in 4 bits: 4.5 GB of codes; the last head's rows lie behind the range of 32-bit byte offsets."""
    m = hp.mk()
    heads, each, last = 7000, 10_000, 300
    total = heads * each + last
    cache = m.MxCache.empty(total, 128)
    g = torch.Generator(device="cuda").manual_seed(1)
    tail = slice(total - last, total)
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t[tail] = torch.randint(0, 256, (last, t.shape[1]), generator=g, device="cuda", dtype=torch.uint8)
    weights = torch.zeros(total, device="cuda")
    weights[tail] = torch.rand(last, generator=g, device="cuda")
    weights[123] = 2.0
    budgets = np.zeros(heads + 1, dtype=np.int32)
    budgets[0], budgets[-1] = 1, 100
    out = m.MxCache.empty(101, 128)
    rows, w, cu_out = (torch.zeros(k, dtype=t, device="cuda") for k, t in ((101, torch.int32), (101, torch.float32), (heads + 2, torch.int32)))
    m.maskkv_evict_mx(mh.desc(1, heads + 1, 128, "bf16", 1, each), weights, mh.device(mh.prefix([each] * heads + [last])), total,
                      mh.device(budgets), cache, None, out, None, rows, w, cu_out, 101)
    assert cu_out.tolist() == [0] + [1] * heads + [101] and rows[0].item() == 123
    want = total - last + np.sort(mxo.stay(weights[tail].cpu().numpy(), 100))
    assert np.array_equal(rows[1:].cpu().numpy(), want)
    at = mh.device(want)
    assert torch.equal(out.k_codes[1:], cache.k_codes[at]) and torch.equal(out.v_scales[1:], cache.v_scales[at])
    assert torch.equal(out.v_codes[1:], cache.v_codes[at]) and torch.equal(w[1:], weights[at])


def test_shapes_are_held_against_the_description():
    m = hp.mk()
    d = mh.desc(1, 2, 64, "bf16", 4, 10)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    i = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")
    f = lambda k: torch.zeros(k, device="cuda")
    good = [d, f(10), mh.device(mh.prefix([4, 6])), 10, i(2) + 3, bf(10, 64), bf(10, 64), i(10), bf(6, 64), bf(6, 64), i(6), i(6), f(6), i(3), 6]
    m.maskkv_evict(*good)
    torch.cuda.synchronize()
    for at, x in ((1, f(9)), (1, i(10)), (2, i(2)), (4, i(1)), (5, bf(9, 64)), (6, f(640)), (7, i(9)), (8, bf(5, 64)), (10, i(5)), (11, i(5)),
                  (12, f(5)), (13, i(2)), (3, 11), (14, 7)):
        with pytest.raises((AssertionError, TypeError)):
            m.maskkv_evict(*(x if k == at else a for k, a in enumerate(good)))
    for at, x in ((8, good[5]), (12, good[1]), (11, good[7]), (13, good[2]), (10, good[11])):        # buffers that overlap
        with pytest.raises(m.MaskKVError):
            m.maskkv_evict(*(x if k == at else a for k, a in enumerate(good)))
    with pytest.raises(m.MaskKVError):
        m.maskkv_evict(*(None if k == 7 else a for k, a in enumerate(good)))                          # idx_out without idx
