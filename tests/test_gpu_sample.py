"""maskkv_sample against the float64 definition (needs an MI355X).

Tokens are compared as numbers.  The device's masses are off by 1e-13 and the oracle's sums by less; a draw that lies within 1e-10 of the mass of where it would
come out otherwise, or a limit, would be left out of the comparison, and the tests say how many were (none may be more than one in a thousand).

prob is a quotient of two 64-bit masses, rounded to 32 bits.  logprob: a term of the sum is off by 3 u of its distance to the largest logit (the difference, the product with log2 e and its
constant) and 2 ulp; 32 terms of a lane are added in 32 bits, the rest in 64; the quotient is rounded once."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu

U = mh.U


class Case:
    def __init__(self, logits, dtype="f32", T=1.0, k=None, p=None, m=None, u=None, seed=0, stride=None, shift=0):
        self.mk, rng = hp.mk(), np.random.default_rng(seed)
        x = torch.from_numpy(np.ascontiguousarray(logits, dtype=np.float32)).to(hp.torch_dtype(dtype))
        self.l = x.float().numpy()
        self.rows, self.V = self.l.shape
        stride = self.V if stride is None else stride
        room = torch.full((self.rows * stride + shift + 8,), float("nan"), dtype=x.dtype, device="cuda")
        self.logits = room[shift:shift + self.rows * stride].view(self.rows, stride)[:, :self.V]
        self.logits.copy_(x.cuda())
        each = lambda v, t: None if v is None else np.broadcast_to(np.asarray(v, dtype=t), (self.rows,)).copy()
        self.T, self.k, self.p, self.m = each(T, np.float32), each(k, np.int32), each(p, np.float32), each(m, np.float32)
        self.u = each(rng.random(self.rows) if u is None else u, np.float32)
        self.given = [None if v is None else mh.device(v) for v in (self.T, self.k, self.p, self.m, self.u)]
        self.token = torch.full((self.rows,), -7, dtype=torch.int32, device="cuda")
        self.prob, self.logprob = torch.full((2, self.rows), 7.0, device="cuda")
        code = self.mk.MASKKV_BF16 if dtype == "bf16" else self.mk.MASKKV_F32
        self.ws = hp.workspace(self.mk.maskkv_sample_workspace_bytes(self.rows, self.V, code))
        self.ws.fill_(255)

    def run(self, stream=None):
        self.mk.maskkv_sample(self.logits, *self.given, self.token, self.prob, self.logprob, self.ws, stream)
        return self

    def check(self, rows=None):
        torch.cuda.synchronize()
        token, prob, logprob = self.token.cpu().numpy(), self.prob.double().cpu().numpy(), self.logprob.double().cpu().numpy()
        rows = range(self.rows) if rows is None else rows
        near = 0
        for r in rows:
            at = lambda v, none: none if v is None else v[r]
            want, p, lp, margin = do.sample(self.l[r], at(self.T, 1.0), at(self.k, 0), at(self.p, 1.0), at(self.m, 0.0), self.u[r])
            if margin < 1e-10 and token[r] != want:
                near += 1
                continue
            assert token[r] == want, f"row {r}: token {token[r]}, not {want} (margin {margin:.1e})"
            assert abs(prob[r] - p) <= 1.02 * U * p + 1e-12, f"row {r}: prob {prob[r]}, not {p}"
            if lp == -np.inf:
                assert logprob[r] == -np.inf
                continue
            l = np.where(np.isnan(self.l[r]), -np.inf, self.l[r].astype(np.float64))
            if l.max() == np.inf:
                l = np.where(l == np.inf, 0.0, -np.inf)
            far = (l.max() - l)[l > -np.inf]
            share = np.exp(-far) / np.exp(-far).sum()
            bound = (share * (3 * U * far + 4 * U)).sum() + 35 * U + abs(lp) * 1.02 * U + 1e-12
            assert abs(logprob[r] - lp) <= bound, f"row {r}: logprob {logprob[r]}, not {lp} ({abs(logprob[r] - lp):.1e}, {bound:.1e} allowed)"
        assert near <= len(rows) / 1000
        return self


def rows_of(rng, rows, V, sharp=True, spread=2.0):
    l = rng.standard_normal((rows, V)) * spread
    if sharp:
        for r in range(rows):
            l[r, rng.integers(0, V, 24)] += 8.0 + 3.0 * rng.standard_normal(24)
    return l


LIMITS = [dict(), dict(k=5), dict(p=0.9), dict(m=0.05), dict(k=50, p=0.9), dict(k=40, p=0.8, m=0.02), dict(k=1), dict(p=0.0), dict(m=1.0), dict(p=0.999, m=1e-6),
          dict(k=100000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("limits", LIMITS, ids=str)
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 2049, 32001])
def test_limits_and_sizes(dtype, limits, V):
    rng = np.random.default_rng(V)
    rows = 9 if V > 2000 else 40
    for sharp in (True, False):
        Case(rows_of(rng, rows, V, sharp), dtype, T=0.5 + rng.random(rows), seed=V, **limits).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [0.0, -1.0, 1e-3, 0.2, 1.0, 3.0, 1e6, float("inf"), float("nan"), 1e-40])
def test_temperatures(dtype, T):
    rng = np.random.default_rng(5)
    l = rows_of(rng, 20, 5000)
    for limits in (dict(), dict(k=30, p=0.95), dict(m=0.1)):
        Case(l, dtype, T=T, seed=6, **limits).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("limits", [dict(), dict(p=0.7), dict(p=0.995), dict(p=0.9, m=1e-5), dict(k=70000), dict(k=3000, p=0.9), dict(m=0.01), dict(p=0.99, m=0.3)], ids=str)
def test_nearly_flat_rows_of_many_tokens(dtype, limits):
    rng = np.random.default_rng(7)
    V = 126464 if dtype == "bf16" else 80001
    l = np.concatenate((rng.standard_normal((2, V)) * 0.5, rng.standard_normal((2, V)) * 3.0))
    Case(l, dtype, T=1.3, seed=8, **limits).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V", [(16, 30000), (40, 9001), (290, 5000)])
def test_many_rows_of_which_most_are_nearly_flat(dtype, rows, V):
    """Among them some of equal logits, some with a few
    values, and some with other limits; each gives the bits that it gives alone."""
    rng = np.random.default_rng(rows)
    l = rng.standard_normal((rows, V)) * np.where(rng.random((rows, 1)) < 0.5, 0.3, 2.0)
    l[3::11] = 1.25
    l[4::11] = rng.integers(0, 4, (len(l[4::11]), V))
    l[5::11, ::7] = -np.inf
    l[6::11, 17] += 30.0
    p = np.where(rng.random(rows) < 0.9, 0.2 + 0.79 * rng.random(rows), 1.0)
    for other in (dict(), dict(k=np.where(rng.random(rows) < 0.2, 40, 0), m=np.where(rng.random(rows) < 0.2, 0.01, 0.0))):
        c = Case(l, dtype, T=0.8 + rng.random(rows), p=p, seed=rows, **other).run().check()
        want = c.token.clone(), c.prob.clone()
        for r in range(0, rows, 5):
            one = Case(l[r:r + 1], dtype, T=c.T[r], p=c.p[r], u=c.u[r], **{n: v[r] for n, v in other.items()}).run()
            torch.cuda.synchronize()
            assert int(one.token[0]) == int(want[0][r]) and float(one.prob[0]) == float(want[1][r])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5, 300, 10007])
def test_ties(dtype, V):
    rng = np.random.default_rng(9)
    l = np.concatenate((np.zeros((6, V)), rng.integers(-2, 3, (6, V))))                 # all equal; five values
    l[3, ::2] = -0.0
    for limits in (dict(), dict(k=3), dict(k=V - 1), dict(p=0.4), dict(k=V // 2 + 1, p=0.77), dict(m=1.0), dict(m=0.5)):
        Case(l, dtype, T=0.9, seed=10, **limits).run().check()


@pytest.mark.parametrize("limits", [dict(), dict(k=2), dict(p=0.6), dict(m=0.2), dict(T=0.0), dict(k=50, p=0.6, m=0.01)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_nan_and_rows_without_a_token(dtype, limits):
    rng = np.random.default_rng(11)
    l = rows_of(rng, 12, 3000)
    l[0] = -np.inf
    l[1] = np.nan
    l[2, ::2] = -np.inf
    l[3, ::3] = np.nan
    l[4, [5, 100, 2999]] = np.inf
    l[5] = np.inf
    l[6, 1:] = -np.inf
    l[7, :-1] = np.nan
    l[8, 17] = np.inf
    l[9] = 3e38
    l[10, 10:20] = -3e38
    l[10, 20] = 3e38
    l[11, rng.integers(0, 3000, 700)] = -np.inf
    Case(l, dtype, seed=12, **limits).run().check()


def test_random_numbers_at_and_beyond_their_ends():
    rng = np.random.default_rng(13)
    l = rows_of(rng, 8, 700)
    u = [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, np.nan, np.inf, 2.0 ** -24]
    for limits in (dict(), dict(k=9), dict(p=0.5), dict(m=0.001)):
        Case(l, "f32", u=u, **limits).run().check()
    # a token whose mass is nothing is never drawn, at either end
    l = np.full((2, 100), -np.inf)
    l[:, [40, 41]] = 0.0
    c = Case(l, "f32", u=[0.0, 1.0]).run().check()
    assert c.token.tolist() == [40, 41]


def test_limits_that_are_none():
    rng = np.random.default_rng(14)
    l = rows_of(rng, 6, 900)
    a = Case(l, seed=15, k=[0, -3, 900, 5000, 2 ** 31 - 1, -2 ** 31], p=[1.0, 2.0, np.nan, np.inf, 1.0, 1.5], m=[0.0, -1.0, np.nan, -np.inf, -0.0, 0.0]).run().check()
    b = Case(l, seed=15, T=None).run().check()
    torch.cuda.synchronize()
    assert torch.equal(a.token, b.token) and torch.equal(a.prob, b.prob) and torch.equal(a.logprob, b.logprob)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,stride,shift", [(1001, 1001, 0), (1001, 1003, 1), (4097, 4100, 3), (5, 5, 1), (2048, 2056, 5), (17, 64, 7)])
def test_rows_that_begin_anywhere(dtype, V, stride, shift):
    """Rows of an odd number of logits behind each other; what lies beside them is NaN."""
    rng = np.random.default_rng(16)
    for limits in (dict(), dict(k=7, p=0.9), dict(p=0.9)):
        Case(rows_of(rng, 13, V), dtype, stride=stride, shift=shift, seed=17, **limits).run().check()


def test_every_row_has_its_own_limits():
    rng = np.random.default_rng(18)
    rows, V = 300, 4000
    l = rows_of(rng, rows, V, spread=2.0)
    l[::3] = rng.standard_normal((100, V))
    c = Case(l, "bf16", T=np.where(rng.random(rows) < 0.1, 0, 0.2 + 1.5 * rng.random(rows)), k=np.where(rng.random(rows) < 0.5, rng.integers(1, 3000, rows), 0),
             p=np.where(rng.random(rows) < 0.5, rng.random(rows), 1.0), m=np.where(rng.random(rows) < 0.3, 0.3 * rng.random(rows), 0.0), seed=19)
    c.run().check()
    want = c.token.clone(), c.prob.clone(), c.logprob.clone()
    c.prob = c.logprob = None                                    # what is not asked for changes nothing
    c.token.zero_()
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.token, want[0])


def test_draws_follow_the_distribution():
    rng = np.random.default_rng(20)
    l = np.tile(rng.standard_normal((1, 50)), (4000, 1))
    c = Case(l, "f32", T=0.8, k=20, u=(np.arange(4000) + 0.5) / 4000).run().check(rows=range(0, 4000, 50))
    counts = np.bincount(c.token.cpu().numpy(), minlength=50) / 4000
    w = np.exp(c.l[0].astype(np.float64) / np.float32(0.8))
    w[np.argsort(-w)[20:]] = 0
    assert np.abs(counts - w / w.sum()).max() <= 1.01 / 4000


def test_many_parts():
    """A row of many millions of logits: more parts than a workgroup has threads."""
    rng = np.random.default_rng(21)
    V = (1 << 24) - 3
    l = rng.standard_normal((1, V)).astype(np.float32)
    l[0, 12345678] += 14
    for limits in (dict(), dict(k=20), dict(p=0.5), dict(m=0.3)):
        Case(l, "bf16", T=0.7, u=0.77, **limits).run().check()


@pytest.mark.parametrize("limits", [dict(), dict(k=50, p=0.9), dict(p=0.97), dict(p=0.9, T=1.5)], ids=str)
def test_captured_replayed_and_equal_bits(limits):
    rng = np.random.default_rng(22)
    c = Case(rows_of(rng, 30, 20000, sharp=False), "bf16", seed=23, **limits).run()
    torch.cuda.synchronize()
    outputs = lambda: (c.token, c.prob, c.logprob)
    want = [x.clone() for x in outputs()]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.run()
    for _ in range(3):
        for x in outputs():
            x.zero_()
        c.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    c.check()


def test_random_rows():
    rng = np.random.default_rng(24)
    for i in range(30):
        V = int(np.exp(rng.uniform(0, 11)))
        limits = {n: v for n, v in (("k", int(np.exp(rng.uniform(0, 8)))), ("p", float(rng.random())), ("m", float(np.exp(rng.uniform(-9, 0))))) if rng.random() < 0.5}
        Case(rows_of(rng, int(rng.integers(1, 12)), V, rng.random() < 0.6, float(rng.uniform(0.1, 4))), str(rng.choice(["bf16", "f32"])),
             T=float(np.exp(rng.uniform(-2, 1.5))), seed=400 + i, **limits).run().check()
