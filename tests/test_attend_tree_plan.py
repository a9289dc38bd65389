"""How maskkv_attend_tree deals a cache out (CPU): which shapes take which form - the kernel of 32 or of 128 query rows, a head whole or its keys dealt to several
workgroups, their partial results joined in either way - and that a workspace is as large as a call needs."""
import numpy as np
import pytest

# name: dtype, B, H, g, d, n, rows of the heads; query rows of a workgroup, whether keys are dealt out, whether a workgroup joins a row.
FORMS = {}


def form(name, dtype, B, H, g, d, n, lens, tile_rows, dealt, shared):
    FORMS[name] = (dtype, B, H, g, d, n, lens, tile_rows, dealt, shared)


def ragged(count, most, seed, **more):
    """Lengths of `count` heads, up to `most`, with some empty ones."""
    rng = np.random.default_rng(seed)
    lens = np.exp(rng.uniform(0, np.log(most + 1), count)).astype(int)
    lens[::5] = 0
    lens[-1] = most
    for at, n in more.items():
        lens[int(at[1:])] = n
    return [int(x) for x in lens]


for _d in (64, 128):
    form(f"32 rows, whole heads, {_d}", "bf16", 2, 3, 2, _d, 20, [0, 100, 33, 64, 1, 31], 32, False, False)
    form(f"32 rows, dealt, {_d}", "bf16", 1, 4, 1, _d, 40, [2500, 0, 700, 2501], 32, True, False)
    form(f"32 rows, dealt, joined by workgroups, {_d}", "bf16", 1, 1, 7, _d, 1, [6001], 32, True, True)
    form(f"32 rows, response over several units, {_d}", "bf16", 1, 3, 1, _d, 300, [3000, 0, 2000], 32, True, False)
    form(f"fp32, whole heads, {_d}", "f32", 2, 12, 3, _d, 130, [40, 0, 5, 33, 1, 64, 31, 32] * 3, 32, False, False)
    form(f"fp32, dealt, {_d}", "f32", 1, 3, 1, _d, 130, [700, 0, 100], 32, True, False)
    form(f"fp32, dealt, joined by workgroups, {_d}", "f32", 1, 1, 1, _d, 5, [6001], 32, True, True)
    form(f"128 rows, whole heads, {_d}", "bf16", 3, 8, 7, _d, 130, ragged(24, 130, 1, h3=64, h4=128, h6=1, h7=129), 128, False, False)
    form(f"128 rows, whole heads, a tile of response, {_d}", "bf16", 1, 64, 7, _d, 60, ragged(64, 64, 2), 128, False, False)
    form(f"128 rows, dealt, {_d}", "bf16", 2, 4, 2, _d, 130, [3000, 0, 428, 2993, 2944, 2945, 2999, 2816], 128, True, False)
    form(f"128 rows, dealt, joined by workgroups, {_d}", "bf16", 1, 4, 2, _d, 150, [9000, 0, 8986, 1285], 128, True, True)
    form(f"128 rows, response over several units, {_d}", "bf16", 1, 1, 3, _d, 900, [2500], 128, True, False)


def plan_of(name):
    from paper_2510_09309_amd import bench_binding as bb
    from paper_2510_09309_amd import binding as mk
    dtype, B, H, g, d, n, lens = FORMS[name][:7]
    desc = mk.Desc(B=B, H=H, d=d, dtype=mk.MASKKV_BF16 if dtype == "bf16" else mk.MASKKV_F32, n_resp=n, P_max=max(lens), q_per_kv=0 if g == 1 else g)
    return bb.maskkv_bench_attend_tree_plan(desc, sum(lens))


@pytest.mark.parametrize("name", FORMS)
def test_the_form_of_every_case(name):
    p = plan_of(name)
    assert (p.tile_rows, p.chunk > 0, bool(p.shared)) == FORMS[name][7:], p
    if "several units" in name:
        tile = 64 if p.tile_rows == 128 else 32
        assert -(-FORMS[name][5] // tile) > p.chunk, p


def descriptions(seed, count):
    from paper_2510_09309_amd import binding as mk
    rng = np.random.default_rng(seed)
    for _ in range(count):
        yield rng, mk.Desc(B=int(rng.integers(1, 9)), H=int(np.exp(rng.uniform(0, 4.5))), d=int(rng.choice([64, 128])), dtype=int(rng.integers(0, 2)),
                           n_resp=int(np.exp(rng.uniform(0, 7))), P_max=int(np.exp(rng.uniform(0, 13))), q_per_kv=int(rng.choice([0, 2, 7])))


def test_a_workspace_holds_what_every_smaller_cache_needs():
    from paper_2510_09309_amd import bench_binding as bb
    from paper_2510_09309_amd import binding as mk
    needed = 0
    for rng, desc in descriptions(0, 1500):
        capacity = int(np.exp(rng.uniform(0, 16)))
        room = mk.maskkv_attend_tree_workspace_bytes(desc, capacity)
        for c in (capacity, 0, *(int(capacity * x) for x in rng.random(6)), *(int(capacity ** x) for x in rng.random(6))):
            needs = bb.maskkv_bench_attend_tree_plan(desc, c).needs
            assert needs <= room, (desc, capacity, c)
            needed += needs > 0
    assert needed > 1000


def test_no_cache_has_more_units_than_there_is_room_for():
    """Heads of any lengths whose sum is the capacity at most."""
    from paper_2510_09309_amd import bench_binding as bb
    dealt = 0
    for rng, desc in descriptions(1, 3000):
        heads = desc.B * desc.H
        lens = np.minimum(np.exp(rng.uniform(0, np.log(desc.P_max + 1), heads)).astype(np.int64) * (rng.random(heads) < 0.8), desc.P_max)
        if rng.random() < 0.3:
            lens[:] = int(rng.integers(0, desc.P_max + 1))
        p = bb.maskkv_bench_attend_tree_plan(desc, min(int(lens.sum()), (1 << 31) - (1 << 17)))
        tile = 64 if p.tile_rows == 128 else 32
        assert p.qtiles * p.tile_rows >= desc.n_resp * max(desc.q_per_kv, 1)
        if not p.chunk:
            assert p.units == heads and p.needs == 0
            continue
        units = -(-(-(-lens // tile) + -(-desc.n_resp // tile)) // p.chunk)
        assert units.min() >= 1 and units.sum() <= p.units
        dealt += 1
    assert dealt > 500
