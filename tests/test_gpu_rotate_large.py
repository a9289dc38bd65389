"""maskkv_rotate of tensors so large that it writes (128 MB and more read and written) or reads and writes (512 MB) past the memory-side cache (needs an MI355X).

Each row is what a call of a few tokens, which does neither, makes of it, bit for bit; some rows of it are compared with the definition."""
import numpy as np
import pytest
import torch

from tests import helpers as hp
from tests import mx_helpers as mh
from tests.test_gpu_rotate import check
from oracle import decode_oracle as do

pytestmark = pytest.mark.gpu

MB = 1 << 20


@pytest.mark.parametrize("order", ["bhtd", "bthd"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,width,place", [(150, 128, "out"), (150, 96, "in"), (540, 64, "out"), (540, 128, "in")])
def test_large_tensors(dtype, layout, order, size, width, place):
    m, B, H, g, d = hp.mk(), 2, 2, 3, 128
    eb = 2 if dtype == "bf16" else 4
    T = -(-size * MB // (2 * B * H * (g + 1) * d * eb)) + 13
    lens = [T, T - 11]                                           # (rows behind a sequence's last one stay as they are)
    assert 2 * B * T * H * (g + 1) * d * eb >= (128 if size == 150 else 512) * MB and (size != 150 or 2 * B * T * H * (g + 1) * d * eb < 512 * MB)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(size + width)

    def room(heads):
        t = torch.randn((B, heads, T, d) if order == "bhtd" else (B, T, heads, d), generator=gen, device="cuda").to(hp.torch_dtype(dtype))
        return t if order == "bhtd" else t.transpose(1, 2)

    Q, K = room(H * g), room(H)
    desc = mh.desc(B, H, d, dtype, 1, 0, g)
    r = m.maskkv_rotary_frequencies(width, 0 if layout == "halves" else 1)
    pos = (torch.arange(T, device="cuda", dtype=torch.int32) + torch.tensor([[5], [100000]], dtype=torch.int32, device="cuda")).contiguous()
    rng = np.random.default_rng(size)
    at = [0, T - 64] + [int(x) for x in rng.integers(0, T - 64, 20)]
    want = []
    for a in at:                                                 # 64 tokens a call
        q, k = torch.empty((B, H * g, 64, d), dtype=Q.dtype, device="cuda"), torch.empty((B, H, 64, d), dtype=Q.dtype, device="cuda")
        m.maskkv_rotate(desc, r, pos[:, a:a + 64].contiguous(), 64, Q[:, :, a:a + 64], q, K[:, :, a:a + 64], k)
        want.append((q, k))
    behind = [x[1, :, lens[1]:].clone() for x in (Q, K)]
    before = Q[1, :, at[2]:at[2] + 64].double().cpu().numpy()
    if place == "out":
        Qo, Ko = torch.full_like(Q, 7.0), torch.full_like(K, 7.0)
        behind = [torch.full_like(x, 7.0) for x in behind]
    else:
        Qo, Ko = Q, K
    m.maskkv_rotate(desc, r, pos, T, Q, Qo, K, Ko, token_len=lens)
    torch.cuda.synchronize()
    for a, (q, k) in zip(at, want):
        for out, x in ((Qo, q), (Ko, k)):
            for b in range(B):
                n = min(64, lens[b] - a)
                assert torch.equal(out[b, :, a:a + n], x[b, :, :n]), (a, b)
    assert torch.equal(Qo[1, :, lens[1]:], behind[0]) and torch.equal(Ko[1, :, lens[1]:], behind[1])
    n = min(64, lens[1] - at[2])
    freq, amplitude = do.frequencies(width, 10000.0)
    check(Qo[1, :, at[2]:at[2] + n].double().cpu().numpy(), before[:, :n], pos[1, at[2]:at[2] + n].cpu().numpy(), freq, amplitude, width, layout, dtype)
