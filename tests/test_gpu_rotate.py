"""maskkv_rotate against the float64 definition (needs an MI355X).

Error bound, u = 2^-24: what is left of an angle after whole turns is rounded to 32 bits, by 2^-26 turns (half a step below 1/2), 1.6 u as radians and less than
2 u; sine and cosine are off by at most 4 u and their product with the amplitude by another u: 7 u of what they multiply.  Two products and a
sum add 3 u of the magnitudes.  The angle's own roundings (frequency in turns, product; the oracle has them in radians) are 4 * 2^-53 of it.  The result is rounded to its dtype."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu

U = mh.U


def check(got, x, positions, freq, amplitude, width, layout, dtype, tag=""):
    want = do.rotate(x, positions, freq, amplitude, width, layout)
    half = width // 2
    most = np.zeros(x.shape)
    i = np.arange(half)
    a, b = (i, i + half) if layout == "halves" else (2 * i, 2 * i + 1)
    both = np.abs(x[..., a].astype(np.float64)) + np.abs(x[..., b].astype(np.float64))
    turn = np.abs(np.asarray(positions, dtype=np.float64))[:, None] * freq
    most[..., a] = most[..., b] = amplitude * both * (10 * U + turn * 4 * 2.0 ** -53)
    bound = most + np.abs(want) * mh.HALF[dtype] * 1.02 + 1e-38
    bound[..., width:] = 0.0                                     # (moved as they are)
    off = np.abs(got - want)
    assert np.all(off <= bound), f"{tag}: {(off / np.maximum(bound, 1e-300)).max():.2f} times the bound off"


class Case:
    def __init__(self, seed, B, H, d, T, width, layout="halves", g=1, dtype="bf16", order="bhtd", scaling="plain", factor=1.0, far=1000, pad=0):
        self.m, rng = hp.mk(), np.random.default_rng(seed)
        self.B, self.H, self.d, self.T, self.g, self.dtype, self.width, self.layout = B, H, d, T, g, dtype, width, layout
        self.q, self.k = mh.gauss(rng, B, H * g, T, d, dtype=dtype), mh.gauss(rng, B, H, T, d, dtype=dtype)
        self.positions = rng.integers(-far, far + 1, (B, T)).astype(np.int32)
        self.desc = mh.desc(B, H, d, dtype, 1, 0, g)
        names = {"plain": 0, "linear": 1, "base": 2, "bands": 3}
        self.rotary = self.m.maskkv_rotary_frequencies(width, 0 if layout == "halves" else 1, 10000.0, names[scaling], factor, 4096.0)
        self.freq, self.amplitude = do.frequencies(width, 10000.0, scaling, factor, 4096.0)
        self.order, self.pad = order, pad
        self.Q, self.K = self.room(H * g, self.q), self.room(H, self.k)
        self.Qo, self.Ko = self.room(H * g), self.room(H)
        self.pos = mh.device(self.positions)

    def room(self, heads, fill=None):
        """[B, heads, T, d] of any order, with `pad` elements (a multiple of 16 bytes) between a row and the next."""
        shape = (self.B, heads, self.T, self.d + self.pad) if self.order == "bhtd" else (self.B, self.T, heads, self.d + self.pad)
        t = torch.full(shape, 7.0, dtype=hp.torch_dtype(self.dtype), device="cuda")
        t = t[..., :self.d] if self.order == "bhtd" else t[..., :self.d].transpose(1, 2)
        if fill is not None:
            t.copy_(hp.upload(fill, self.dtype))
        return t

    def run(self, stream=None, **kw):
        self.m.maskkv_rotate(self.desc, self.rotary, self.pos, self.T, self.Q, self.Qo, self.K, self.Ko, stream, **kw)

    def check(self, tag="", sides=("Q", "K")):
        torch.cuda.synchronize()
        for name, out, x in (("Q", self.Qo, self.q), ("K", self.Ko, self.k)):
            got = out.double().cpu().numpy()
            for b in range(self.B if name in sides else 0):
                check(got[b], x[b], self.positions[b], self.freq, self.amplitude, self.width, self.layout, self.dtype, f"{tag} {name} {b}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("d,width", [(64, 64), (128, 128), (128, 64), (64, 48), (128, 80), (64, 8), (128, 36), (64, 6), (128, 2), (128, 126), (64, 4)])
def test_widths_and_layouts(dtype, layout, d, width):
    c = Case(1, 2, 3, d, 11, width, layout, g=2, dtype=dtype)
    c.run()
    c.check()


@pytest.mark.parametrize("T", [1, 2, 3, 7, 8, 9, 64, 1000])
@pytest.mark.parametrize("B,H,g", [(1, 1, 1), (3, 4, 7), (2, 32, 1), (64, 1, 1)])
def test_lengths_and_heads(T, B, H, g):
    if B * H * g * T > 70000:
        T = 333
    c = Case(2, B, H, 128 if H < 32 else 64, T, 64, g=g, order="bthd" if T % 2 else "bhtd")
    c.run()
    c.check()


@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("base", 8.0), ("bands", 4.0), ("bands", 1.0)])
def test_scaled_frequencies(scaling, factor):
    for dtype in ("bf16", "f32"):
        c = Case(3, 1, 2, 128, 65, 128, dtype=dtype, scaling=scaling, factor=factor, far=40000)
        c.run()
        c.check()


@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 1])
def test_far_positions(far):
    c = Case(4, 1, 2, 128, 200, 128, dtype="f32", far=far)
    c.positions[0, :2] = (-2 ** 31, 2 ** 31 - 1) if far > 1 << 20 else (0, far)
    c.pos = mh.device(c.positions)
    c.run()
    c.check()


@pytest.mark.parametrize("order", ["bhtd", "bthd"])
@pytest.mark.parametrize("dtype,pad", [("bf16", 8), ("f32", 4)])
def test_strides_and_what_lies_between_rows(order, dtype, pad):
    c = Case(5, 2, 3, 64, 21, 40, "pairs", g=2, dtype=dtype, order=order, pad=pad)
    c.run()
    c.check()
    for t in (c.Qo, c.Ko):
        whole = t.transpose(1, 2)._base if order == "bthd" else t._base
        assert bool((whole[..., 64:] == 7.0).all())


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("width", [128, 48, 10])
def test_in_place_and_back(layout, width):
    c = Case(6, 2, 2, 128, 50, width, layout, g=3, dtype="f32")
    c.run()
    c.Qo, c.Ko, out = c.Q, c.K, (c.Qo, c.Ko)
    c.run()
    c.check("in place")
    assert torch.equal(c.Q, out[0]) and torch.equal(c.K, out[1])
    c.pos = mh.device(-c.positions)
    c.run()
    torch.cuda.synchronize()
    # (two rotations: each off by 10 u of two elements' magnitudes at amplitude 1)
    assert float((c.Q.cpu() - torch.from_numpy(c.q)).abs().max()) <= 2 * 10 * U * 2 * np.abs(c.q).max() + 2 * U * np.abs(c.q).max()


def test_one_side_only_and_lengths_of_sequences():
    c = Case(7, 4, 2, 64, 30, 64, g=2)
    lens = [30, 0, 7, 1]
    c.run(token_len=lens)
    torch.cuda.synchronize()
    for out, x in ((c.Qo, c.q), (c.Ko, c.k)):
        got = out.double().cpu().numpy()
        for b, n in enumerate(lens):
            check(got[b, :, :n], x[b, :, :n], c.positions[b, :n], c.freq, c.amplitude, 64, "halves", "bf16")
            assert np.all(got[b, :, n:] == 7.0)                  # rows behind a sequence's last one
    c.Qo.fill_(7.0)
    c.Ko.fill_(7.0)
    c.m.maskkv_rotate(c.desc, c.rotary, c.pos, c.T, None, None, c.K, c.Ko)
    c.check(sides=("K",))
    assert bool((c.Qo == 7.0).all())
    c.Ko.fill_(7.0)
    c.m.maskkv_rotate(c.desc, c.rotary, c.pos, c.T, c.Q, c.Qo, None, None)
    c.check(sides=("Q",))
    assert bool((c.Ko == 7.0).all())
    c.Qo.fill_(7.0)
    c.run(token_len=[0] * 4)
    torch.cuda.synchronize()
    assert bool((c.Qo == 7.0).all())


def test_packed_sequences_and_the_rows_of_a_cache():
    """Sequences behind each other on one axis; and a packed cache as one sequence of one head, moved to other positions."""
    m, rng = hp.mk(), np.random.default_rng(8)
    lens, start = [5, 17, 1], [0, 5, 22]
    x = mh.gauss(rng, 1, 2, 23, 64)
    pos = np.zeros((3, 17), dtype=np.int32)
    for b, n in enumerate(lens):
        pos[b, :n] = np.arange(n) + 100 * b
    K = hp.upload(x, "bf16")
    out = torch.zeros_like(K)
    v = lambda t: m.tensor_view(t.expand(3, -1, -1, -1), seq_start=start)
    r = m.maskkv_rotary_frequencies(64)
    m.maskkv_rotate(mh.desc(3, 2, 64, "bf16", 1, 0), r, mh.device(pos), 17, None, None, v(K), v(out), token_len=lens)
    torch.cuda.synchronize()
    freq, amplitude = do.frequencies(64, 10000.0)
    got = out.double().cpu().numpy()[0]
    for b, n in enumerate(lens):
        check(got[:, start[b]:start[b] + n], x[0, :, start[b]:start[b] + n], pos[b, :n], freq, amplitude, 64, "halves", "bf16")
    cache = mh.gauss(rng, 700, 64)
    idx = np.sort(rng.choice(5000, 700, replace=False)).astype(np.int32)
    Kc = hp.upload(cache, "bf16").view(1, 1, 700, 64)
    m.maskkv_rotate(mh.desc(1, 1, 64, "bf16", 1, 0), r, mh.device(idx), 700, None, None, Kc, Kc)
    torch.cuda.synchronize()
    check(Kc.double().cpu().numpy()[0, 0], cache, idx, freq, amplitude, 64, "halves", "bf16")


def test_infinities_and_nan_stay_in_their_pairs():
    c = Case(9, 1, 1, 64, 4, 32, dtype="f32")
    c.Q[0, 0, 1, 3], c.Q[0, 0, 2, 40] = float("nan"), float("inf")
    c.run()
    torch.cuda.synchronize()
    got = c.Qo[0, 0].cpu().numpy()
    bad = np.zeros((4, 64), dtype=bool)
    bad[1, [3, 19]] = True
    assert np.array_equal(np.isnan(got), bad) and got[2, 40] == np.inf


def test_captured_and_replayed_on_another_stream():
    c = Case(10, 2, 4, 128, 77, 128, g=2)
    c.run()
    torch.cuda.synchronize()
    want = [c.Qo.clone(), c.Ko.clone()]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.run()
    for _ in range(3):
        c.Qo.zero_(), c.Ko.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.Qo, want[0]) and torch.equal(c.Ko, want[1])
    c.Qo.zero_()
    torch.cuda.synchronize()
    c.run(side)
    torch.cuda.synchronize()
    assert torch.equal(c.Qo, want[0])


def test_a_large_tensor_behind_4_gib():
    m = hp.mk()
    T = (1 << 24) + 1000                                          # 4.3 GB of 128 bf16
    x = torch.zeros((1, 1, T, 128), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(11)
    tail = mh.gauss(rng, 1, 1, 1000, 128)
    x[:, :, -1000:] = hp.upload(tail, "bf16")
    pos = torch.arange(T, dtype=torch.int32, device="cuda").view(1, T)
    m.maskkv_rotate(mh.desc(1, 1, 128, "bf16", 1, 0), m.maskkv_rotary_frequencies(128), pos, T, None, None, x, x)
    torch.cuda.synchronize()
    freq, amplitude = do.frequencies(128, 10000.0)
    check(x[0, 0, -1000:].double().cpu().numpy(), tail[0, 0], np.arange(T - 1000, T), freq, amplitude, 128, "halves", "bf16")
    assert float(x[0, 0, :1000].abs().max()) == 0.0


def test_random_shapes():
    rng = np.random.default_rng(12)
    for i in range(40):
        d = int(rng.choice([64, 128]))
        c = Case(100 + i, int(rng.integers(1, 6)), int(rng.integers(1, 13)), d, int(np.exp(rng.uniform(0, 6))), 2 * int(rng.integers(1, d // 2 + 1)),
                 str(rng.choice(["halves", "pairs"])), int(rng.choice([1, 1, 3, 7])), str(rng.choice(["bf16", "f32"])), str(rng.choice(["bhtd", "bthd"])),
                 str(rng.choice(["plain", "linear", "base", "bands"])), float(rng.uniform(1, 9)), int(np.exp(rng.uniform(0, 14))), pad=8 * int(rng.integers(0, 2)))
        c.run()
        c.check(f"case {i}")
