"""maskkv_tree_mask and maskkv_attend_tree against the float64 definitions (needs an MI355X)."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu

U = mh.U


# ---- masks
def random_parents(rng, B, n, gone=0.0):
    p = np.array([[int(rng.integers(max(-1, i - 6), i)) if i else -1 for i in range(n)] for _ in range(B)], dtype=np.int32).reshape(B, n)
    return np.where(rng.random((B, n)) < gone, -2, p).astype(np.int32)


def masks(parents):
    m = hp.mk()
    B, n = parents.shape
    out = torch.full((B, n, (n + 31) // 32), -1, dtype=torch.int32, device="cuda")
    m.maskkv_tree_mask(mh.device(parents), out)
    torch.cuda.synchronize()
    return out.cpu().numpy().view(np.uint32)


@pytest.mark.parametrize("B,n", [(1, 1), (3, 2), (2, 31), (2, 32), (5, 33), (64, 64), (1, 257), (3, 600), (1, 5000)])
def test_masks_of_trees(B, n):
    rng = np.random.default_rng(n)
    for parents in ([random_parents(rng, B, n), random_parents(rng, B, n, 0.2), np.tile(np.arange(-1, n - 1, dtype=np.int32), (B, 1))] if n < 1000
                    else [random_parents(rng, B, n)]):
        got = masks(parents)
        for b in range(B):
            assert np.array_equal(got[b], do.words(do.tree(parents[b])))


def test_masks_of_parents_that_are_none():
    n = 70
    rng = np.random.default_rng(3)
    parents = rng.integers(-2 ** 31, 2 ** 31, (4, n)).astype(np.int32)          # anything at all
    parents[1] = rng.integers(-3, n + 3, n)
    parents[2] = np.arange(n)                                                   # itself
    parents[3] = -2
    got = masks(parents)
    for b in range(4):
        assert np.array_equal(got[b], do.words(do.tree(parents[b])))
    assert not got[3].any()


# ---- attention
class Case:
    def __init__(self, seed, B, H, d, n, lens, g=1, dtype="bf16", sees="tree", spare=0, size=1.0, P_max=None):
        self.m, rng = hp.mk(), np.random.default_rng(seed)
        self.rng, self.B, self.H, self.d, self.n, self.g, self.dtype = rng, B, H, d, n, g, dtype
        lens = [int(x) for x in (lens if hasattr(lens, "__len__") else [lens] * (B * H))]
        self.lens, self.cu, self.cap = lens, mh.prefix(lens), sum(lens) + spare
        self.q, self.k, self.v = (mh.gauss(rng, *s, dtype=dtype, size=size) for s in ((B, H * g, n, d), (self.cap, d), (self.cap, d)))
        self.kr, self.vr = mh.gauss(rng, B, H, n, d, dtype=dtype, size=size), mh.gauss(rng, B, H, n, d, dtype=dtype)
        self.sees = self.who(sees)
        self.desc = mh.desc(B, H, d, dtype, n, max(lens) if P_max is None else P_max, g)
        self.upload()

    def who(self, sees):
        B, n = self.B, self.n
        if sees == "tree":
            return np.stack([do.tree(p) for p in random_parents(self.rng, B, n)])
        if sees == "blocks":
            b = np.arange(n) // 8
            return np.broadcast_to(b[:, None] >= b[None, :], (B, n, n)).copy()
        if sees == "any":                                        # rows that see nothing among them
            return self.rng.random((B, n, n)) < self.rng.random((B, n, 1)) * (self.rng.random((B, n, 1)) < 0.8)
        return np.full((B, n, n), sees == "all")

    def upload(self):
        up = lambda x: hp.upload(x, self.dtype)
        self.Q, self.K, self.V, self.Kr, self.Vr = (up(x) for x in (self.q, self.k, self.v, self.kr, self.vr))
        self.CU = mh.device(self.cu)
        self.mask = mh.device(np.stack([do.words(s) for s in self.sees]).view(np.int32))
        self.O, self.lse = torch.full_like(self.Q, 7.0), torch.full((self.B * self.H * self.g * self.n,), 7.0, device="cuda")
        self.ws = hp.workspace(self.m.maskkv_attend_tree_workspace_bytes(self.desc, self.cap))
        if self.ws is not None:
            self.ws.fill_(255)                                   # (NaN)

    def run(self, stream=None, scale=0.0, capacity=None, ws="own"):
        self.m.maskkv_attend_tree(self.desc, self.Q, self.K, self.V, self.CU, self.cap if capacity is None else capacity, self.Kr, self.Vr, self.mask, scale,
                                  self.O, self.lse, self.ws if isinstance(ws, str) else ws, stream)
        return self

    def check(self, scale=None, heads=None, capacity=None):
        """The bound of the other attentions over a packed cache: a probability is off by twice a logit's error and, as the operand of the
        second product, by half a step of the dtype; the sums by a rounding a key; the result by half a step."""
        torch.cuda.synchronize()
        O, lse = self.O.double().cpu().numpy(), self.lse.double().cpu().numpy().reshape(self.B * self.H, self.g, self.n)
        scale = 1.0 / np.sqrt(self.d) if scale is None else scale
        capacity = self.cap if capacity is None else capacity
        half = mh.HALF[self.dtype]
        for i in range(self.B * self.H) if heads is None else heads:
            b, h = i // self.H, i % self.H
            a, z = min(self.cu[i], capacity), min(self.cu[i + 1], capacity)
            q = self.q[b, h * self.g:(h + 1) * self.g]
            want, norm, mass = do.attend(q, self.k[a:z], self.v[a:z], self.kr[b, h], self.vr[b, h], self.sees[b], scale)
            got, gl = O[b, h * self.g:(h + 1) * self.g], lse[i]
            some = np.isfinite(norm)
            assert np.all(got[~some & (norm == -np.inf)] == 0.0) and np.all(gl[norm == -np.inf] == -np.inf), f"head {i}: rows that see nothing"
            if not some.any():
                continue
            keys = np.concatenate((self.k[a:z], self.kr[b, h]))
            e = mh.logit_error(q.reshape(-1, self.d), np.nan_to_num(keys, posinf=0, neginf=0), scale, norm[some])
            n = z - a + self.n
            bound = mass * (2 * e + 2 * (n + 40) * U + half * 1.02) + np.abs(want) * half * 1.02 + 1e-30
            with np.errstate(invalid="ignore"):
                off = np.where(np.isnan(want), 0.0, np.abs(got - want) / bound)[some]
            off = np.where(np.isinf(want[some]) & (got[some] == want[some]), 0.0, off)
            assert np.array_equal(np.isnan(got[some]), np.isnan(want[some])), f"head {i}: NaN"
            assert off.max() <= 1.0, f"head {i}: an output is {off.max():.2f} times its bound off"
            far = np.abs(gl[some] - norm[some]).max()
            assert far <= 2 * e + (n + 40) * U, f"head {i}: a normaliser is {far:.3e} off"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 8, 31, 32, 33, 65])
def test_small(dtype, d, n):
    Case(n, 2, 2, d, n, [0, 1, 40, 33], dtype=dtype).run().check()


@pytest.mark.parametrize("sees", ["tree", "blocks", "any", "all", "none"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_who_sees_whom(sees, dtype):
    c = Case(20, 2, 3, 64, 100, [0, 7, 64, 300, 0, 31], g=2, dtype=dtype, sees=sees).run()
    c.check()


@pytest.mark.parametrize("n,g,H,rows", [(1, 7, 4, 9000), (1, 1, 2, 30011), (5, 3, 1, 20001), (48, 7, 1, 3001), (64, 1, 3, 4096), (33, 1, 2, 2000), (130, 1, 2, 1500),
                                        (96, 7, 1, 700)])
def test_few_rows_over_long_heads(n, g, H, rows):
    c = Case(21, 1, H, 128, n, rows, g=g)
    c.run().check()


def test_heads_of_very_different_lengths_dealt_out():
    rng = np.random.default_rng(22)
    lens = np.exp(rng.uniform(0, 9, 12)).astype(int)
    lens[3], lens[7] = 0, 12000
    for dtype in ("bf16", "f32"):
        Case(22, 3, 4, 64, 9, lens, dtype=dtype, g=2, sees="any").run().check()


def test_many_heads():
    rng = np.random.default_rng(23)
    c = Case(23, 16, 40, 64, 3, rng.integers(0, 90, 640))
    c.run().check(heads=range(0, 640, 37))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,rows", [(6, 40), (40, 100), (70, 0), (6, 9000), (140, 300)])
def test_infinities_and_nan_in_what_a_row_does_not_see(dtype, n, rows):
    c = Case(24, 1, 2, 64, n, rows, dtype=dtype, g=2)
    bad = [0, n // 2, n - 1]
    for j, x in zip(bad, (np.nan, np.inf, -np.inf)):
        c.sees[:, :, j] = False
        c.sees[:, j, j] = False
        c.kr[:, :, j], c.vr[:, :, j] = x, x
    c.sees[:, 1, bad[0]] = True                                   # one row sees a NaN,
    c.upload()
    c.run().check()
    O = c.O.float().cpu().numpy()
    assert np.isnan(O[:, :, 1]).all()
    assert np.isfinite(np.delete(O, 1, axis=2)).all()
    c.kr = np.nan_to_num(c.kr, nan=0.5, posinf=0.5, neginf=0.5)   # and now one an infinite value with finite logits
    c.sees[:, 1, bad[0]] = False
    c.sees[:, 2, bad[1]] = True
    c.vr[:, :, bad[1], ::2] = -np.inf
    c.upload()
    c.run().check()
    O = c.O.float().cpu().numpy()
    assert (O[:, :, 2, ::2] == -np.inf).all() and (O[:, :, 2, 1::2] == np.inf).all()
    assert np.isfinite(np.delete(O, 2, axis=2)).all()


@pytest.mark.parametrize("n", [3, 33, 100, 200])
def test_rows_of_other_heads_and_beyond_the_cache_do_not_reach_a_head(n):
    """NaN in the rows behind the last head, in a head of its own between two others, and in what lies behind the response's rows."""
    c = Case(25, 1, 3, 64, n, [50, 20, 41], spare=40, sees="any")
    c.k[50:70], c.v[50:70] = np.nan, np.nan
    c.k[111:], c.v[111:] = np.nan, np.nan
    c.upload()
    wide = torch.full((1, 3, n + 40, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    for name in ("Kr", "Vr"):
        w = wide.clone()
        w[:, :, :n] = getattr(c, name)
        setattr(c, name, w[:, :, :n])
    c.run().check(heads=(0, 2))
    assert bool(torch.isnan(c.O[:, 1]).all())


def test_bits_behind_the_last_row_are_not_looked_at():
    c = Case(26, 1, 2, 64, 37, 20, sees="any")
    c.run()
    want = c.O.clone()
    c.mask[..., 1] |= ~0x1F                                       # columns 37 .. 63
    c.O.zero_()
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.O, want)


@pytest.mark.parametrize("size", [6.0, 30.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(size, dtype):
    Case(27, 1, 2, 64, 20, [700, 33], dtype=dtype, size=size).run().check()


def test_a_scale_and_no_normalisers():
    c = Case(28, 1, 2, 128, 12, 200)
    c.run(scale=0.02).check(scale=np.float64(np.float32(0.02)))
    want = c.O.clone()
    lse, c.lse = c.lse, None
    c.O.zero_()
    c.run(scale=0.02)
    torch.cuda.synchronize()
    assert torch.equal(c.O, want)


def test_the_capacity_cuts_off_rows_and_an_empty_cache():
    c = Case(29, 1, 3, 64, 10, [40, 50, 60])
    c.run(capacity=70).check(capacity=70)
    c = Case(30, 1, 2, 64, 40, [0, 0])
    c.K = c.V = None
    c.run().check()


@pytest.mark.parametrize("order", ["bthd", "padded"])
def test_strides(order):
    c = Case(31, 2, 2, 64, 40, [100, 0, 5, 70], g=3, sees="blocks")

    def other(t):
        if order == "bthd":
            return t.transpose(1, 2).contiguous().transpose(1, 2)
        w = torch.full((t.shape[0], t.shape[1], t.shape[2] + 3, t.shape[3] + 8), 7.0, dtype=t.dtype, device="cuda")
        w[:, :, :t.shape[2], :t.shape[3]] = t
        return w[:, :, :t.shape[2], :t.shape[3]]

    c.Q, c.Kr, c.Vr, c.O = (other(t) for t in (c.Q, c.Kr, c.Vr, c.O))
    c.run().check()
    if order == "padded":
        assert bool((c.O._base[:, :, 40:] == 7.0).all() and (c.O._base[..., 64:] == 7.0).all())


def test_it_is_the_unmasked_attention_where_all_is_seen():
    c = Case(32, 2, 2, 128, 70, [300, 20, 0, 900], sees="all").run()
    O = torch.zeros_like(c.O)
    lse = torch.zeros_like(c.lse)
    c.m.maskkv_attend(c.desc, c.Q, c.K, c.V, c.CU, c.cap, c.Kr, c.Vr, 0.0, O, lse, hp.workspace(c.m.maskkv_attend_workspace_bytes(c.desc, False)))
    torch.cuda.synchronize()
    # (both within their bound of the definition: logits of order 1, outputs below 5)
    assert float((O.float() - c.O.float()).abs().max()) <= 2e-2 and float((lse - c.lse).abs().max()) <= 1e-4


def test_positions_beyond_2_gib_of_rows():
    """A head whose rows lie behind 4 GiB of others."""
    m = hp.mk()
    before = (1 << 25) + 5                                        # rows of 128 bytes: 4.3 GB of K, and of V
    c = Case(33, 1, 2, 64, 4, [0, 300])
    big = lambda x: torch.cat((torch.zeros((before, 64), dtype=torch.bfloat16, device="cuda"), x))
    c.K, c.V = big(c.K), big(c.V)
    c.CU = mh.device(np.array([0, before, before + 300], dtype=np.int32))
    c.desc = mh.desc(1, 2, 64, "bf16", 4, before)
    c.ws = hp.workspace(m.maskkv_attend_tree_workspace_bytes(c.desc, before + 300))
    c.run(capacity=before + 300)
    c.check(heads=(1,))


@pytest.mark.parametrize("kw", [dict(n=64, lens=4000), dict(n=1, g=7, lens=9000), dict(n=6, lens=50, dtype="f32"), dict(n=150, lens=600)])
def test_captured_replayed_and_equal_bits(kw):
    c = Case(34, 1, 2, 64, **kw).run()
    torch.cuda.synchronize()
    want = (c.O.clone(), c.lse.clone())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.run()
    for _ in range(3):
        c.O.zero_(), c.lse.zero_()
        if c.ws is not None:
            c.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.O, want[0]) and torch.equal(c.lse, want[1])


def test_a_shrinking_cache_keeps_its_workspace():
    c = Case(35, 1, 2, 64, 2, 40000, P_max=40000)
    ws = c.ws
    for rows in (30000, 9000, 2000, 300, 10, 0):
        s = Case(36, 1, 2, 64, 2, rows, P_max=40000)
        s.run(ws=ws).check()


def test_random_shapes():
    rng = np.random.default_rng(37)
    for i in range(40):
        B, H, g, n = int(rng.integers(1, 4)), int(rng.integers(1, 6)), int(rng.choice([1, 1, 2, 7])), int(np.exp(rng.uniform(0, 5)))
        lens = np.exp(rng.uniform(0, rng.uniform(1, 7.5), B * H)).astype(int) * (rng.random(B * H) < 0.9)
        c = Case(300 + i, B, H, int(rng.choice([64, 128])), n, lens, g, str(rng.choice(["bf16", "bf16", "f32"])), str(rng.choice(["tree", "blocks", "any"])),
                 P_max=int(lens.max() + rng.integers(0, 5000)))
        c.run().check()
