"""Caches without rows, held in tensors without elements (which have no address), through every call that takes them."""
import numpy as np
import pytest
import torch

from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu

HEADS, D = 3, 64


def room(*shape, dtype=torch.float32, fill=7):
    return torch.full(shape, fill, dtype=dtype, device="cuda")


def rows_of(m, mx, n):
    return (m.MxCache.empty(n, D),) if mx else (room(n, D, dtype=torch.bfloat16), room(n, D, dtype=torch.bfloat16))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("with_idx", [False, True])
@pytest.mark.parametrize("n,n_out", [(0, 0), (0, 5), (6, 0)])
def test_eviction_from_and_into_a_cache_without_rows(mx, with_idx, n, n_out):
    """Positions are passed on both sides, or on neither; where there are no rows they are an empty tensor."""
    m = hp.mk()
    lens = [n // 3] * HEADS
    idx, idx_out = (room(k, dtype=torch.int32) if with_idx else None for k in (n, n_out))
    rows, w_out, cu_out = room(n_out, dtype=torch.int32), room(n_out), room(HEADS + 1, dtype=torch.int32)
    budgets = mh.device(np.array([1, 0, 2], dtype=np.int32))
    call = m.maskkv_evict_mx if mx else m.maskkv_evict
    call(mh.desc(1, HEADS, D, "bf16", 1, 10), torch.rand(n, device="cuda"), mh.device(mh.prefix(lens)), n, budgets, *rows_of(m, mx, n), idx,
         *rows_of(m, mx, n_out), idx_out, rows, w_out, cu_out, n_out)
    torch.cuda.synchronize()
    stay = np.minimum([1, 0, 2], lens)
    assert cu_out.tolist() == mh.prefix(stay).tolist()
    for x in (rows, w_out, idx_out):
        assert x is None or (x == 7).all()                     # nothing was there to be written


def test_eviction_still_needs_positions_on_both_sides_where_rows_may_move():
    m = hp.mk()
    for mx in (False, True):
        call = m.maskkv_evict_mx if mx else m.maskkv_evict
        for idx, idx_out in ((room(6, dtype=torch.int32), None), (None, room(5, dtype=torch.int32))):
            with pytest.raises(m.MaskKVError) as e:
                call(mh.desc(1, HEADS, D, "bf16", 1, 10), room(6), mh.device(mh.prefix([2, 2, 2])), 6, room(HEADS, dtype=torch.int32, fill=1),
                     *rows_of(m, mx, 6), idx, *rows_of(m, mx, 5), idx_out, room(5, dtype=torch.int32), None, room(HEADS + 1, dtype=torch.int32), 5)
            assert e.value.status == 1


@pytest.mark.parametrize("n", [1, 20, 200])
def test_the_other_calls_on_a_cache_without_rows(n):
    m = hp.mk()
    desc = mh.desc(1, HEADS, D, "bf16", n, 10)
    rng = np.random.default_rng(n)
    Q, K, V = (mh.gauss(rng, 1, HEADS, n, D) for _ in range(3))
    up = lambda x: hp.upload(x, "bf16")
    cu, cache, plain = mh.device(mh.prefix([0, 0, 0])), m.MxCache.empty(0, D), room(0, D, dtype=torch.bfloat16)
    idx = room(0, dtype=torch.int32)
    prompt = room(1, HEADS, 10, D, dtype=torch.bfloat16)
    m.maskkv_compact_mx(desc, prompt, prompt, idx, cu, 0, cache)
    m.maskkv_expand_mx(desc, cache, cu, 0, plain, plain)
    O, lse = torch.zeros(1, HEADS, n, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(HEADS * n, device="cuda")
    ws = hp.workspace(m.maskkv_attend_mx_workspace_bytes(desc, 0))
    m.maskkv_attend_mx(desc, up(Q), cache, cu, 0, up(K), up(V), 0.0, O, lse, ws)
    for decay in (0.0, 0.5):
        m.maskkv_accumulate_mx(desc, up(Q), cache, cu, 0, 0.0, lse, decay, room(0), room(0))
        m.maskkv_accumulate(desc, up(Q), plain, cu, 0, 0.0, lse, decay, room(0), room(0))
    torch.cuda.synchronize()
    for h in range(HEADS):
        mh.check_attention(O[0, h].double().cpu().numpy(), lse.view(HEADS, n)[h].double().cpu().numpy(), Q[0, h], K[0, h], V[0, h], "bf16")
