"""A cache that shrinks keeps the workspace that was allocated for it at first."""
import numpy as np
import pytest
import torch

from tests import helpers as hp
from tests import mx_helpers as mh
from tests.test_gpu_attend_mx import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,g,n,d,sizes", [(1, 4, 7, 1, 128, (131072, 91750, 40000, 500)), (1, 8, 1, 32, 128, (15564, 14745, 3000, 0)),
                                             (2, 2, 4, 100, 64, (47513, 42598, 9000))])
def test_one_workspace_for_all_later_sizes(B, H, g, n, d, sizes):
    m = hp.mk()
    c = Case(50 + n, B, H, d, "bf16", n, [sizes[0] // (B * H)] * (B * H), g=g)
    desc = mh.desc(B, H, d, "bf16", n, c.P_max, g)
    ws = hp.workspace(m.maskkv_attend_mx_workspace_bytes(desc, sizes[0]))
    cache = mh.cache(c.K, c.V, spare=B * H)
    up = lambda x: hp.upload(x, "bf16")
    Q, Kr, Vr = up(c.Q), up(c.Kr), up(c.Vr)
    for size in sizes:
        c.cu = mh.prefix([size // (B * H)] * (B * H))
        O = torch.full((B, H * g, n, d), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((B * H * g * n,), 7.0, device="cuda")
        if ws is not None:
            ws.fill_(255)
        m.maskkv_attend_mx(desc, Q, cache, mh.device(c.cu), size, Kr, Vr, 0.0, O, lse, ws)
        torch.cuda.synchronize()
        c.O, c.lse = O.double().cpu().numpy(), lse.double().cpu().numpy().reshape(B * H, -1)
        c.check(heads=[0, B * H - 1])
