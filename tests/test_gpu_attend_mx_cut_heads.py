"""maskkv_attend_mx where only heads of more than so many tiles are cut: what is left of them are units of their own, and are joined."""
import numpy as np
import pytest
import torch

from tests import helpers as hp
from tests import mx_helpers as mh
from tests.test_gpu_attend_mx import Case

pytestmark = pytest.mark.gpu
LONG = 1 << 20


def plan(H, d, n, capacity, B=1):
    from paper_2510_09309_amd import bench_binding as bb
    p = bb.maskkv_bench_attend_mx_plan(mh.desc(B, H, d, "bf16", n, LONG), capacity)
    assert p.tile_rows == 128 and p.ranked and p.extras > 0, p
    return p, -(-n // 64)                                             # its response tiles


def case(seed, B, H, d, n, lens):
    c = Case(seed, B, H, d, "bf16", n, lens)
    c.P_max = LONG
    return c


@pytest.mark.parametrize("B,H,d,n,capacity", [(1, 200, 128, 200, 60000), (2, 100, 64, 300, 100000), (1, 256, 128, 129, 80000), (4, 64, 128, 257, 80000)])
def test_heads_around_the_length_from_which_they_are_cut(B, H, d, n, capacity):
    p, resp = plan(B * H // B, d, n, capacity, B)
    rows = lambda tiles: (tiles - resp) * 64
    C = p.chunk
    lens = np.random.default_rng(H + d).integers(0, 60, B * H)
    special = {0: rows(C), 1: rows(C) + 1, 5: rows(2 * C), 63: rows(2 * C) + 1, 64: rows(C) - 63, 100: 0, 130: rows(5 * C) + 17, B * H - 1: rows(C) + 64}
    for at, k in special.items():
        lens[at] = k
    assert lens.sum() <= capacity
    run = case(60, B, H, d, n, lens.tolist()).run(capacity=capacity)
    run.check(heads=sorted(special) + [2, 62, 99, 180])


@pytest.mark.parametrize("H,d,n,capacity", [(200, 128, 200, 40000), (200, 64, 300, 100000)])
def test_as_many_cut_heads_as_there_is_room_for(H, d, n, capacity):
    """Most places of the workspace are used; the last head is clipped by the capacity, where it comes to that."""
    p, resp = plan(H, d, n, capacity)
    least = (p.chunk - resp) * 64 + 1
    many = min(capacity // least, H)
    lens = [0] * H
    for i in range(many):
        lens[i * H // many] = least
    lens[H - 1] += 500                                                # behind the capacity, all or in part
    c = case(61, 1, H, d, n, lens)
    c.run(capacity=capacity).check(capacity=capacity, heads=[0, 1, H // many, (many // 2) * H // many, H - 2, H - 1])
    assert p.cut * 0.6 < many <= p.cut


def test_one_head_that_has_nearly_all_rows():
    p, _ = plan(256, 128, 200, 60000)
    lens = [3] * 256
    lens[77] = 58000
    case(62, 1, 256, 128, 200, lens).run(capacity=60000).check(heads=[0, 76, 77, 78, 255])


def test_replays_and_two_streams():
    """Partial results of a call in a graph and of one beside it, each with a workspace of its own that holds anything before."""
    m = hp.mk()
    H, d, n, capacity = 200, 128, 200, 60000
    p, _ = plan(H, d, n, capacity)
    programs = []
    for seed in (63, 64):
        lens = np.random.default_rng(seed).integers(0, 60, H)
        lens[[seed % 7, 150]] = [9000, 7000 + seed]
        c = case(seed, 1, H, d, n, lens.tolist())
        desc = mh.desc(1, H, d, "bf16", n, LONG)
        cache, cu = mh.cache(c.K, c.V, spare=capacity - int(c.cu[-1])), mh.device(c.cu)
        Q, Kr, Vr = (hp.upload(x, "bf16") for x in (c.Q, c.Kr, c.Vr))
        O, lse = torch.zeros(1, H, n, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(H * n, device="cuda")
        ws = hp.workspace(m.maskkv_attend_mx_workspace_bytes(desc, capacity))

        def call(stream=None, a=(desc, Q, cache, cu, capacity, Kr, Vr, 0.0, O, lse, ws)):
            m.maskkv_attend_mx(*a, stream)
        call()
        torch.cuda.synchronize()
        c.O, c.lse = O.double().cpu().numpy(), lse.double().cpu().numpy().reshape(H, n)
        c.check(heads=[seed % 7, 8, 150])
        programs.append((call, O, lse, ws, O.clone(), lse.clone()))
    graphs = []
    for call, *_ in programs:
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            call()
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for replay in range(3):
        for call, O, lse, ws, *_ in programs:
            O.zero_(), lse.zero_(), ws.fill_(255)
        torch.cuda.synchronize()
        for graph, (call, *_), stream in zip(graphs, programs, streams):
            if replay == 2:
                call(stream)
            else:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for _, O, lse, _, O_want, lse_want in programs:
            assert torch.equal(O, O_want) and torch.equal(lse, lse_want), f"replay {replay}"
