"""How maskkv_attend_mx deals out a cache whose prompt was long (CPU): heads x query tiles that fill the chip are not cut into pieces because one
of them might hold all of the prompt."""
import pytest


@pytest.fixture(scope="module")
def plan():
    from paper_2510_09309_amd import bench_binding as bb
    from paper_2510_09309_amd import binding as mk

    def of(B, H, d, n, rows, P_max, g=0):
        desc = mk.Desc(B=B, H=H, d=d, dtype=mk.MASKKV_BF16, n_resp=n, P_max=P_max, q_per_kv=g)
        return bb.maskkv_bench_attend_mx_plan(desc, rows), mk.maskkv_attend_mx_workspace_bytes(desc, rows)
    return of


@pytest.mark.parametrize("B,H,d,n,rows", [(8, 32, 128, 512, 88845), (4, 32, 128, 512, 44517), (8, 32, 128, 256, 55228), (8, 32, 64, 512, 88845),
                                          (2, 100, 128, 200, 78329)])
def test_the_longest_prompt_says_nothing_of_the_heads_of_an_evicted_cache(plan, B, H, d, n, rows):
    short, none = plan(B, H, d, n, rows, 16384)
    assert short.tile_rows == 128 and short.chunk == 0 and short.ranked and none == 0
    tiles = rows / 64 / (B * H) + -(-n // 64)                       # of a head on average
    for P_max in (32768, 131072, 1 << 20):
        p, size = plan(B, H, d, n, rows, P_max)
        assert p.tile_rows == 128 and p.ranked and p.extras > 0     # whole heads by length, but for those that take longest
        assert p.chunk >= 2 * tiles
        assert size <= 25 << 20                                      # (all heads dealt out: 16 ... 103 MB)


def test_no_head_is_cut_where_there_is_no_room_for_a_long_one(plan):
    p, size = plan(8, 32, 128, 512, 15000, 1 << 20)
    assert p.tile_rows == 128 and p.chunk == 0 and p.ranked
