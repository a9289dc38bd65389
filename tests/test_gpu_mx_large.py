"""Caches in 4 bits of so many rows that counts of bytes, or of threads, pass 32 bits."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mxo
from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu


def needs(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"{gib} GiB of device memory are not free")


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def test_rows_whose_threads_pass_32_bits():
    """2^28 + 77 rows of 128 fp32 or bf16: 16 threads a row store them (fp32) and expand them, 2^32 are more than a launch has along
    a dimension.  All rows but the last ones are row 0 of a prompt."""
    needs(175)
    m = hp.mk()
    rng = np.random.default_rng(1)
    n, d, P, last = (1 << 28) + 77, 128, 50, 1000
    x = mh.gauss(rng, 2, P, d)                                                          # values that bf16 and fp32 hold
    idx = torch.zeros(n, dtype=torch.int32, device="cuda")
    tail = rng.integers(0, P, last).astype(np.int32)
    idx[n - last:] = mh.device(tail)
    at = np.concatenate(([0, 0], tail))
    look = torch.cat((torch.tensor([0, n // 2], device="cuda"), torch.arange(n - last, n, device="cuda")))
    cu = mh.device(np.array([0, 5, n], dtype=np.int32))                                  # two heads with the same prompt
    cache = m.MxCache.empty(n, d)
    for dtype in ("f32", "bf16"):
        desc = mh.desc(1, 2, d, dtype, 1, P)
        K, V = (hp.upload(np.stack((y, y))[None], dtype) for y in x)
        for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
            t[look] = 0xA5
        m.maskkv_compact_mx(desc, K, V, idx, cu, n, cache)
        torch.cuda.synchronize()
        for y, codes, scales in ((x[0], cache.k_codes, cache.k_scales), (x[1], cache.v_codes, cache.v_scales)):
            want = mxo.store(y)
            assert np.array_equal(codes[look].cpu().numpy(), want[0][at]) and np.array_equal(scales[look].cpu().numpy(), want[1][at]), dtype
    Kc, Vc = (torch.empty(n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m.maskkv_expand_mx(desc, cache, cu, n, Kc, Vc)
    torch.cuda.synchronize()
    for y, out in ((x[0], Kc), (x[1], Vc)):
        assert np.array_equal(out[look].float().cpu().numpy(), mh.stored(y)[at].astype(np.float32))


def test_accumulating_over_rows_whose_threads_pass_32_bits():
    """2^31 - 65536 rows of 64 over 600 heads: 128 rows a workgroup of 256 threads, and one more of them a head."""
    needs(100)
    m = hp.mk()
    heads, d, n = 600, 64, 0x7FFF0000
    rng = np.random.default_rng(2)
    codes = torch.zeros(n, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, d // 32), 127, dtype=torch.uint8, device="cuda")
    some = 300                                                                           # rows of every head but the second
    lens = np.full(heads, some, dtype=np.int64)
    lens[1] = n - some * (heads - 1)
    cu = mh.prefix(lens)
    K = mh.gauss(rng, some, d)
    want = mxo.store(K)
    for i in (0, heads - 1):
        codes[cu[i]:cu[i] + some], scales[cu[i]:cu[i] + some] = mh.device(want[0]), mh.device(want[1])
    Q = mh.gauss(rng, 1, heads, 1, d)
    lse = np.full((heads, 1), 2.0, dtype=np.float32)
    out = torch.full((n,), 7.0, device="cuda")
    m.maskkv_accumulate_mx(mh.desc(1, heads, d, "bf16", 1, 1 << 29), hp.upload(Q, "bf16"), m.MxCache(codes, scales), mh.device(cu), n, 0.0,
                           mh.device(lse.ravel()), 0.0, None, out)
    torch.cuda.synchronize()
    for i in (0, heads - 1):
        got = out[cu[i]:cu[i + 1]].double().cpu().numpy()
        mh.check_weights(got, Q[0, i], mh.stored(K), lse[i].astype(np.float64), 0.0, None, tag=f"head {i}")
    for a, z in ((cu[1], cu[1] + 1000), (cu[2] - 1000, cu[2])):                           # keys of zeros: exp(-2) each
        assert np.abs(out[a:z].double().cpu().numpy() - np.exp(-2.0)).max() < 1e-6


class FarCache:
    """Rows of 128 in 4 bits, 4.5 GB of codes: one head of 70 million rows of zeros but for a few, the last ones among them, and one of
    300 rows behind them, which all lie beyond the range of 32-bit byte offsets."""

    def __init__(self, seed, d=128, rows=70_000_000):
        m, rng = hp.mk(), np.random.default_rng(seed)
        self.d, self.first, self.last = d, rows, 300
        self.total = rows + self.last
        self.cache = m.MxCache.empty(self.total, d)
        for t in (self.cache.k_codes, self.cache.v_codes):
            t.zero_()
        for t in (self.cache.k_scales, self.cache.v_scales):
            t.fill_(127)
        self.at = np.concatenate((np.sort(rng.choice(rows, 20, replace=False)), np.arange(rows - 5, rows)))   # of the first head
        self.K, self.V = (mh.gauss(rng, len(self.at) + self.last, d) for _ in range(2))
        self.K[:len(self.at), 0] = 96.0                        # far above the zeros for queries with an 8 there: e^68 to one
        where = mh.device(np.concatenate((self.at, np.arange(rows, self.total))))
        for x, codes, scales in ((self.K, self.cache.k_codes, self.cache.k_scales), (self.V, self.cache.v_codes, self.cache.v_scales)):
            c, s = mxo.store(x)
            codes[where], scales[where] = mh.device(c), mh.device(s)
        self.K, self.V = mh.stored(self.K), mh.stored(self.V)
        self.cu = mh.prefix([rows, self.last])

    def heads(self):
        n = len(self.at)
        return (self.K[:n], self.V[:n]), (self.K[n:], self.V[n:])


@pytest.mark.parametrize("d,dtype,n,rows", [(128, "bf16", 1, 16), (128, "bf16", 40, 32), (128, "bf16", 200, 128), (128, "f32", 3, 32), (64, "bf16", 2, 16)])
def test_attention_over_rows_beyond_four_gibibytes(d, dtype, n, rows):
    from paper_2510_09309_amd import bench_binding as bb
    needs(40)
    m, rng = hp.mk(), np.random.default_rng(n)
    far = FarCache(n, d, 70_000_000 * 128 // d)
    desc = mh.desc(1, 2, d, dtype, n, 1 << 29)
    assert bb.maskkv_bench_attend_mx_plan(desc, far.total).tile_rows == rows
    Q, Kr, Vr = (mh.gauss(rng, 1, 2, n, d, dtype=dtype) for _ in range(3))
    Q[..., 0] = 8.0
    up = lambda x: hp.upload(x, dtype)
    O, lse = torch.zeros(1, 2, n, d, dtype=hp.torch_dtype(dtype), device="cuda"), torch.zeros(2 * n, device="cuda")
    m.maskkv_attend_mx(desc, up(Q), far.cache, mh.device(far.cu), far.total, up(Kr), up(Vr), 0.0, O, lse,
                       hp.workspace(m.maskkv_attend_mx_workspace_bytes(desc, far.total)))
    torch.cuda.synchronize()
    for h, (K, V) in enumerate(far.heads()):
        mh.check_attention(O[0, h].double().cpu().numpy(), lse.view(2, n)[h].double().cpu().numpy(), Q[0, h], np.concatenate((K, Kr[0, h])),
                           np.concatenate((V, Vr[0, h])), dtype, tag=f"head {h}")


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 40), ("f32", 3)])
def test_accumulating_over_rows_beyond_four_gibibytes(dtype, n):
    needs(40)
    m, rng = hp.mk(), np.random.default_rng(n)
    far = FarCache(n + 7)
    Q = mh.gauss(rng, 1, 2, n, 128, dtype=dtype)
    Q[..., 0] = 8.0
    lse = np.stack([np.full(n, 70.0), rng.uniform(3.0, 9.0, n)]).astype(np.float32)
    out = torch.full((far.total,), 7.0, device="cuda")
    m.maskkv_accumulate_mx(mh.desc(1, 2, 128, dtype, n, 1 << 29), hp.upload(Q, dtype), m.MxCache(far.cache.k_codes, far.cache.k_scales),
                           mh.device(far.cu), far.total, 0.0, mh.device(lse.ravel()), 0.0, None, out)
    torch.cuda.synchronize()
    got = out[mh.device(far.at)], out[far.first:]
    for h, (K, _) in enumerate(far.heads()):
        mh.check_weights(got[h].double().cpu().numpy(), Q[0, h], K, lse[h].astype(np.float64), 0.0, None, tag=f"head {h}")


def test_the_values_of_rows_beyond_four_gibibytes():
    needs(50)
    m, far = hp.mk(), FarCache(3)
    Kc, Vc = (torch.empty(far.total, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m.maskkv_expand_mx(mh.desc(1, 2, 128, "bf16", 1, 1 << 29), far.cache, mh.device(far.cu), far.total, Kc, Vc)
    torch.cuda.synchronize()
    for want, out in ((far.K, Kc), (far.V, Vc)):
        look = torch.cat((out[mh.device(far.at)], out[far.first:]))
        assert np.array_equal(look.float().cpu().numpy(), want.astype(np.float32))
        assert out[far.first - 1000:far.first - 5].count_nonzero() <= 128 * np.count_nonzero(far.at >= far.first - 1000)
