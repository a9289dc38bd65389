"""The cache in 4 bits on the device against the oracle, byte by byte: eviction into it, and the values it stands for."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mxo
from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu


def positions(rng, P, lens, H):
    """Ascending prompt positions of every head's rows."""
    return np.concatenate([np.sort(rng.permutation(P[i // H])[:k]) for i, k in enumerate(lens)] + [np.zeros(0, int)]).astype(np.int32)


def check_compact(K, V, dtype, P, lens, idx, capacity=None, K_arg=None, V_arg=None):
    """K, V: float32 [B, H, T, d].  Rows behind the last one have to stay as they were."""
    m = hp.mk()
    B, H, T, d = K.shape
    cu = mh.prefix(lens)
    total = int(cu[-1])
    capacity = total if capacity is None else capacity
    spare = 5
    cache = m.MxCache.empty(capacity + spare, d)
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t.fill_(0x5A)
    desc = mh.desc(B, H, d, dtype, 4, max(P), prompt_len=None if len(set(P)) == 1 else P)
    padded = np.concatenate((idx, np.zeros(max(capacity - total, 0) + 1, np.int32)))
    m.maskkv_compact_mx(desc, hp.upload(K, dtype) if K_arg is None else K_arg, hp.upload(V, dtype) if V_arg is None else V_arg,
                        mh.device(padded), mh.device(cu), capacity, cache)
    torch.cuda.synchronize()
    written = min(total, capacity)
    heads = np.repeat(np.arange(B * H), lens)[:written]
    at = np.clip(idx[:written], 0, np.maximum(np.array(P)[heads // H] - 1, 0))
    for x, codes, scales in ((K, cache.k_codes, cache.k_scales), (V, cache.v_codes, cache.v_scales)):
        want = mxo.store(x[heads // H, heads % H, at]) if written else (np.zeros((0, d // 2)), np.zeros((0, d // 32)))
        for got, ref in zip((codes.cpu().numpy(), scales.cpu().numpy()), want):
            assert np.array_equal(got[:written], ref)
            assert (got[written:] == 0x5A).all()
    return cache, desc, cu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,P,lens", [
    (1, 1, [1], [1]), (1, 2, [9], [0, 9]), (1, 3, [40], [7, 0, 40]), (2, 2, [100, 37], [33, 1, 0, 37]),
    (3, 5, [300, 1, 64], [300, 17, 31, 32, 33, 1, 0, 1, 1, 0, 64, 63, 2, 5, 8]), (1, 4, [50], [0, 0, 0, 0])])
def test_rows_are_stored_as_defined(dtype, d, B, H, P, lens):
    rng = np.random.default_rng(d + sum(lens))
    size = np.exp2(rng.integers(-12, 12, (B, H, max(P), 1)))
    K, V = (mh.gauss(rng, B, H, max(P), d, dtype=dtype) * size.astype(np.float32) for _ in range(2))
    check_compact(K, V, dtype, P, lens, positions(rng, P, lens, H))


def test_every_bf16_value():
    """All 65536 of them, beside a group's largest element of each exponent's two kinds and alone."""
    bits = np.arange(65536, dtype=np.uint32)
    every = (bits << 16).view(np.float32).copy()
    rows = [every.reshape(1024, 64)]                                   # neighbours in value: the group's scale is their own
    finite = np.where(np.isfinite(every), every, 0.0).astype(np.float32)
    for mantissa in (1.0, 1.5, 1.5078125, 1.9921875):                   # largest elements at and around the border of a scale
        x = finite.reshape(-1, 16)                                      # 16 values of about one size, and one somewhat larger
        top = np.abs(x).max(axis=1)
        with np.errstate(divide="ignore"):
            lead = np.ldexp(mantissa, np.clip(np.where(top > 0, np.floor(np.log2(top)), -100) + 2, -126, 127).astype(int))
        y = np.zeros((x.shape[0], 32), dtype=np.float32)
        y[:, :16], y[:, 20] = x, lead
        rows.append(y.reshape(-1, 64))
    K = np.concatenate(rows)[None, None]
    n = K.shape[2]
    check_compact(K, K[:, :, ::-1].copy(), "bf16", [n], [n], np.arange(n, dtype=np.int32))
    check_compact(K, K[:, :, ::-1].copy(), "f32", [n], [n], np.arange(n, dtype=np.int32))


def test_fp32_values_at_borders():
    """Values a step of fp32 around every rounding border and every scale's border, and numbers below the normal range."""
    rows = []
    for e in (-140, -127, -126, -125, -124, -123, -60, 0, 60, 120, 124, 125, 126):
        border = np.ldexp(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], dtype=np.float64), e).clip(max=3.4e38).astype(np.float32)
        near = np.concatenate([np.nextafter(border, np.float32(0)), border, np.nextafter(border, np.float32(3.4e38))])
        row = np.zeros(64, dtype=np.float32)
        row[:24], row[32:56] = near, -near[::-1]
        rows.append(row)
        rows.append(np.where(np.arange(64) % 32 < 8, row, 0).astype(np.float32))
    K = np.stack(rows)[None, None]
    n = K.shape[2]
    check_compact(K, -K, "f32", [n], [n], np.arange(n, dtype=np.int32))


def test_groups_with_nan_or_infinity_stand_for_nan():
    rng = np.random.default_rng(5)
    K, V = mh.gauss(rng, 1, 2, 20, 128), mh.gauss(rng, 1, 2, 20, 128)
    K[0, 0, 3, 40], K[0, 1, 4, 127], V[0, 0, 3, 0], V[0, 1, 7, 64] = np.nan, np.inf, -np.inf, np.nan
    m = hp.mk()
    for dtype in ("bf16", "f32"):
        cache, desc, cu = check_compact(K, V, dtype, [20], [20, 20], np.tile(np.arange(20, dtype=np.int32), 2))
        Kc, Vc = (torch.zeros(40, 128, dtype=hp.torch_dtype(dtype), device="cuda") for _ in range(2))
        m.maskkv_expand_mx(desc, cache, mh.device(cu), 40, Kc, Vc)
        k = Kc.float().cpu().numpy()
        assert np.isnan(k[3, 32:64]).all() and np.isnan(k[24, 96:]).all() and np.isnan(k).sum() == 64
        assert np.isnan(Vc.float().cpu().numpy()).sum() == 64


@pytest.mark.parametrize("capacity", [0, 1, 29, 30, 31, 500])
def test_a_capacity_that_is_not_the_number_of_rows(capacity):
    rng = np.random.default_rng(capacity)
    K, V = mh.gauss(rng, 1, 3, 40, 64), mh.gauss(rng, 1, 3, 40, 64)
    check_compact(K, V, "bf16", [40], [10, 0, 20], positions(rng, [40], [10, 0, 20], 3), capacity=capacity)


def test_positions_outside_the_prompt_are_clamped():
    rng = np.random.default_rng(6)
    K, V = mh.gauss(rng, 2, 2, 30, 64), mh.gauss(rng, 2, 2, 30, 64)
    idx = np.array([-5, 0, 29, 30, 1 << 30, 11, 10, -(1 << 31)], dtype=np.int32)
    check_compact(K, V, "bf16", [30, 11], [2, 2, 2, 2], idx)


def test_views_of_other_orders_and_packed_sequences():
    m = hp.mk()
    rng = np.random.default_rng(7)
    K, V = mh.gauss(rng, 2, 3, 50, 128), mh.gauss(rng, 2, 3, 50, 128)
    lens = [20, 3, 50, 41, 0, 7]
    idx = positions(rng, [50, 50], lens, 3)
    tokens = lambda x: hp.upload(x.transpose(0, 2, 1, 3).copy(), "bf16").transpose(1, 2)     # [B, T, H, d] in memory
    check_compact(K, V, "bf16", [50, 50], lens, idx, K_arg=tokens(K), V_arg=tokens(V))
    wide = torch.zeros(2, 3, 50, 160, dtype=torch.bfloat16, device="cuda")
    wide[..., 16:144] = hp.upload(K, "bf16")
    check_compact(K, V, "bf16", [50, 50], lens, idx, K_arg=wide[..., 16:144], V_arg=hp.upload(V, "bf16"))
    # packed sequences of 50 and 31 tokens, [T, H, d], behind 3 tokens that belong to nobody
    P, starts = [50, 31], [3, 53]
    flat = np.zeros((84, 3, 128), dtype=np.float32)
    flat[3:53], flat[53:84] = K[0].transpose(1, 0, 2), K[1, :, :31].transpose(1, 0, 2)
    lens = [20, 3, 50, 31, 0, 7]
    t = hp.upload(flat, "bf16").transpose(0, 1)[None].expand(2, -1, -1, -1)
    view = m.tensor_view(t, seq_start=starts)
    check_compact(K, V, "bf16", P, lens, positions(rng, P, lens, 3), K_arg=view, V_arg=hp.upload(V, "bf16"))


def test_more_heads_than_a_wave_searches_at_once():
    rng = np.random.default_rng(8)
    H = 4200
    K, V = mh.gauss(rng, 1, H, 3, 64), mh.gauss(rng, 1, H, 3, 64)
    lens = rng.integers(0, 4, H)
    lens[100:400] = 0
    check_compact(K, V, "bf16", [3], lens.tolist(), positions(rng, [3], lens, H))


def test_prompts_beyond_four_gibibytes():
    m = hp.mk()
    H, P, d = 20, 1 << 20, 128                                             # 5 GiB of K
    K = torch.zeros(1, H, P, d, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(9)
    idx = np.sort(rng.integers(0, P, (H, 4)), axis=1).astype(np.int32)
    idx[:, 3] = P - 1
    x = mh.gauss(rng, H, 4, d)
    for h in range(H):
        K[0, h, mh.device(idx[h]).long()] = hp.upload(x[h], "bf16")
        x[h] = K[0, h, mh.device(idx[h]).long()].float().cpu().numpy()       # (a position may be there twice)
    cache = m.MxCache.empty(4 * H, d)
    m.maskkv_compact_mx(mh.desc(1, H, d, "bf16", 1, P), K, K, mh.device(idx.ravel()), mh.device(mh.prefix([4] * H)), 4 * H, cache)
    codes, scales = mxo.store(x.reshape(-1, d))
    assert np.array_equal(cache.k_codes.cpu().numpy(), codes) and np.array_equal(cache.v_scales.cpu().numpy(), scales)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,capacity", [([1], 1), ([7, 0, 30], 37), ([0, 0], 4), ([33, 100], 90), ([5], 0), ([3, 4], 300)])
def test_expand_gives_the_values(dtype, d, lens, capacity):
    m = hp.mk()
    rng = np.random.default_rng(sum(lens) + d)
    total = sum(lens)
    codes = [rng.integers(0, 256, (capacity, d // 2)).astype(np.uint8) for _ in range(2)]
    scales = [rng.integers(3, 253, (capacity, d // 32)).astype(np.uint8) for _ in range(2)]
    if capacity > 2:
        scales[0][1, 1] = 255
    cache = m.MxCache(*(mh.device(x) for x in (codes[0], scales[0], codes[1], scales[1])))
    out = [torch.full((capacity + 3, d), 7.0, dtype=hp.torch_dtype(dtype), device="cuda") for _ in range(2)]
    m.maskkv_expand_mx(mh.desc(1, len(lens), d, dtype, 1, 1000), cache, mh.device(mh.prefix(lens)), capacity, *out)
    torch.cuda.synchronize()
    rows = min(total, capacity)
    for i in range(2):
        got = out[i].double().cpu().numpy()
        assert np.array_equal(got[:rows], mxo.values(codes[i], scales[i])[:rows], equal_nan=True)
        assert (got[rows:] == 7.0).all()


def test_capacity_is_held_against_the_tensors():
    m = hp.mk()
    d = mh.desc(1, 2, 64, "bf16", 4, 10)
    K = torch.zeros(1, 2, 10, 64, dtype=torch.bfloat16, device="cuda")
    idx, cu = torch.zeros(20, dtype=torch.int32, device="cuda"), mh.device(mh.prefix([5, 5]))
    cache, rows = m.MxCache.empty(10, 64), torch.zeros(10, 64, dtype=torch.bfloat16, device="cuda")
    bad = [lambda: m.maskkv_compact_mx(d, K, K, idx, cu, 11, cache), lambda: m.maskkv_compact_mx(d, K, K, idx[:9], cu, 10, cache),
           lambda: m.maskkv_compact_mx(d, K, K, idx, cu[:2], 10, cache), lambda: m.maskkv_compact_mx(d, K, K, idx.long(), cu, 10, cache),
           lambda: m.maskkv_compact_mx(d, K[:, :, :9], K, idx, cu, 10, cache), lambda: m.maskkv_compact_mx(d, K, K.float(), idx, cu, 10, cache),
           lambda: m.maskkv_compact_mx(d, K, K[:, :1], idx, cu, 10, cache), lambda: m.maskkv_expand_mx(d, cache, cu, 10, rows, rows[:9]),
           lambda: m.maskkv_expand_mx(d, cache, cu, 10, rows.float(), rows), lambda: m.maskkv_expand_mx(d, cache, cu, 11, rows, rows)]
    for call in bad:
        with pytest.raises((AssertionError, TypeError)):
            call()
