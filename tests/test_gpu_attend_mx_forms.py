"""Every form that maskkv_attend_mx may take, by name: each case first asserts that the plan is the form which it is here for
(a change of the cost model could take a case past it)."""
import numpy as np
import pytest

from tests import mx_helpers as mh
from tests.test_gpu_attend_mx import Case

pytestmark = pytest.mark.gpu


def run(c, rows, dealt, ranked=False, shared=False, heads=None):
    from paper_2510_09309_amd import bench_binding as bb
    desc = mh.desc(c.B, c.H, c.d, c.dtype, c.n, c.P_max, c.g)
    p = bb.maskkv_bench_attend_mx_plan(desc, int(c.cu[-1]))
    assert (p.tile_rows, p.chunk > 0, bool(p.ranked), bool(p.shared)) == (rows, dealt, ranked, shared), p
    c.run().check(heads=heads)


def lengths(seed, heads, lo, hi, **more):
    """Random lengths, with some heads of given ones."""
    lens = np.random.default_rng(seed).integers(lo, hi, heads)
    for at, n in more.items():
        lens[int(at[1:])] = n
    return lens.tolist()


@pytest.mark.parametrize("d", [64, 128])
def test_up_to_16_query_rows(d):
    run(Case(31, 1, 1, d, "bf16", 2, [900], g=8), 16, False)
    run(Case(32, 1, 4, d, "bf16", 1, [5000, 3, 0, 9000], g=7), 16, True)
    run(Case(33, 2, 2, d, "bf16", 16, [4000, 9001, 33, 1]), 16, True)
    run(Case(34, 1, 4, d, "bf16", 1, [29999, 0, 30011, 30001], g=7), 16, True, shared=True)


@pytest.mark.parametrize("d", [64, 128])
def test_32_query_rows_a_workgroup(d):
    run(Case(35, 2, 3, d, "bf16", 40, [100, 0, 63, 64, 65, 1]), 32, False)
    run(Case(36, 1, 2, d, "bf16", 40, [5000, 3]), 32, True)
    run(Case(37, 1, 1, d, "bf16", 33, [60000]), 32, True, shared=True)
    run(Case(38, 1, 2, d, "bf16", 300, [24000, 100]), 32, True)
    run(Case(39, 2, 2, d, "f32", 1, [100, 0, 63, 33]), 32, False)
    run(Case(40, 1, 2, d, "f32", 40, [5000, 3]), 32, True, shared=True)
    run(Case(43, 2, 4, d, "f32", 20, [500, 0, 700, 33, 900, 512, 513, 800]), 32, True)


@pytest.mark.parametrize("d,heads,n,special", [(64, 200, 200, dict(h3=1500, h77=1499, h100=0, h101=0, h199=700)), (64, 64, 512, dict(h0=0, h5=900, h63=901)),
                                               (64, 255, 128, dict(h0=1, h64=1200, h254=0)), (128, 240, 200, dict(h3=1500, h100=0, h239=1100)),
                                               (128, 60, 512, dict(h9=0, h59=800)), (128, 256, 129, dict(h1=0, h192=1000, h255=2))])
def test_128_query_rows_a_workgroup_in_the_order_of_the_heads_lengths(d, heads, n, special):
    """Heads fill one to four sets of 64, not all of them whole."""
    lens = lengths(heads, heads, 0, 200, **special)
    at = sorted({0, 63, heads - 1, heads // 2} & set(range(heads)) | {int(k[1:]) for k in special})
    run(Case(heads, 1, heads, d, "bf16", n, lens), 128, False, ranked=True, heads=at)


@pytest.mark.parametrize("d", [64, 128])
def test_128_query_rows_a_workgroup_and_more_heads_than_are_ordered(d):
    run(Case(41, 1, 257, d, "bf16", 130, lengths(41, 257, 0, 100, h0=300, h256=299)), 128, False, heads=[0, 1, 64, 255, 256])


@pytest.mark.parametrize("d,heads,n,lo,hi,shared", [(64, 32, 384, 3000, 5600, False), (128, 12, 512, 6000, 9000, False), (128, 3, 512, 33000, 34001, True)])
def test_128_query_rows_a_workgroup_with_the_keys_dealt_out(d, heads, n, lo, hi, shared):
    run(Case(heads + d, 1, heads, d, "bf16", n, lengths(42, heads, lo, hi, h1=0 if heads > 4 else 32001)), 128, True, shared=shared,
        heads=[0, 1, heads - 1])


def test_128_query_rows_a_workgroup_with_very_long_heads_dealt_out():
    run(Case(44, 1, 3, 64, "bf16", 700, [60000, 500, 59999]), 128, True, shared=True, heads=[1, 2])
