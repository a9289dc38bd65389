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
