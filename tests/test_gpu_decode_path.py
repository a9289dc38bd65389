"""The calls around an answer as a program makes them, one after the other: positions, eviction into a packed cache, a drafted tree and its mask, the
attention of its rows, and a token for each of them (needs an MI355X)."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from oracle import maskkv_oracle as orc
from tests import helpers as hp
from tests import mx_helpers as mh

pytestmark = pytest.mark.gpu


class Program:
    """A layer's prompt keys are rotated and compressed once; then every step drafts a tree, rotates its rows by their depth behind the prompt, attends, and
    samples a token at each of its nodes from logits that are made of the attention's output (columns of it, enlarged: some occur twice)."""

    def __init__(self, seed, B=2, H=3, g=2, d=64, P=900, n=13, keep=120, V=777, steps=2, dtype="bf16"):
        self.m, rng = hp.mk(), np.random.default_rng(seed)
        m = self.m
        self.B, self.H, self.g, self.d, self.P, self.n, self.V, self.steps, self.dtype = B, H, g, d, P, n, V, steps, dtype
        up = lambda x: hp.upload(x, dtype)
        self.k, self.v = mh.gauss(rng, B, H, P, d, dtype=dtype), mh.gauss(rng, B, H, P, d, dtype=dtype)
        self.qm = mh.gauss(rng, B, H * g, 16, d, dtype=dtype)
        self.rows = [[mh.gauss(rng, B, heads, n, d, dtype=dtype) for heads in (H * g, H, H)] for _ in range(steps)]
        self.parents = np.array([[[int(rng.integers(max(-1, i - 4), i)) if i else -1 for i in range(n)] for _ in range(B)] for _ in range(steps)], dtype=np.int32)
        self.parents[:, -1, n - 3:] = -2                          # the last sequence's trees have three rows less
        depth = np.zeros((steps, B, n), dtype=np.int32)
        for s in range(steps):
            for b in range(B):
                for i in range(n):
                    depth[s, b, i] = depth[s, b, self.parents[s, b, i]] + 1 if self.parents[s, b, i] >= 0 else 0
        self.at = (P + depth).astype(np.int32)
        self.columns = rng.integers(0, H * g * d, V).astype(np.int64)
        self.u = rng.random((steps, B * n)).astype(np.float32)
        self.limits = [0.7, 20, 0.9, 0.01]
        # on the device
        code = m.MASKKV_BF16 if dtype == "bf16" else m.MASKKV_F32
        self.rotary = m.maskkv_rotary_frequencies(d, m.ROTARY_HALVES, 10000.0, m.ROTARY_BANDS, 2.0, 512.0)
        self.prompt = m.Desc(B=B, H=H, d=d, dtype=code, n_resp=16, P_max=P, q_per_kv=g)
        self.desc = m.Desc(B=B, H=H, d=d, dtype=code, n_resp=n, P_max=P, q_per_kv=g)
        self.K, self.V_, self.Qm = up(self.k), up(self.v), up(self.qm)
        self.Kfull = torch.zeros((B, H, P + 16, d), dtype=hp.torch_dtype(dtype), device="cuda")
        self.Kfull[:, :, P:] = up(mh.gauss(rng, B, H, 16, d, dtype=dtype))
        self.prompt_at = torch.arange(P, dtype=torch.int32, device="cuda").repeat(B, 1)
        BH, dt = B * H, hp.torch_dtype(dtype)
        zeros = lambda *s, t=dt: torch.zeros(s, dtype=t, device="cuda")
        self.cap = BH * keep
        self.budgets = torch.full((BH,), keep, dtype=torch.int32, device="cuda")
        self.scores, self.idx, self.cu = zeros(BH, P, t=torch.float32), zeros(self.cap, t=torch.int32), zeros(BH + 1, t=torch.int32)
        self.Kc, self.Vc = zeros(self.cap, d), zeros(self.cap, d)
        self.ws = [hp.workspace(x) for x in (m.maskkv_score_workspace_bytes(self.prompt), m.maskkv_select_workspace_bytes(self.prompt),
                                             m.maskkv_attend_tree_workspace_bytes(self.desc, self.cap), m.maskkv_sample_workspace_bytes(B * n, V, m.MASKKV_F32))]
        self.step = []
        for s in range(steps):
            q, k, v = self.rows[s]
            self.step.append(dict(Q=up(q), K=up(k), V=up(v), Qr=zeros(*q.shape), Kr=zeros(*k.shape), at=mh.device(self.at[s]), parents=mh.device(self.parents[s]),
                                  mask=zeros(B, n, (n + 31) // 32, t=torch.int32), O=zeros(*q.shape), lse=zeros(BH * g * n, t=torch.float32),
                                  logits=zeros(B * n, V, t=torch.float32), u=mh.device(self.u[s]), token=zeros(B * n, t=torch.int32),
                                  prob=zeros(B * n, t=torch.float32), logprob=zeros(B * n, t=torch.float32)))
        self.cols = mh.device(self.columns)
        full = lambda x, t: torch.full((B * n,), x, dtype=t, device="cuda")
        self.given = [full(x, t) for x, t in zip(self.limits, (torch.float32, torch.int32, torch.float32, torch.float32))]

    def run(self, stream=None):
        m, B, H, g, n = self.m, self.B, self.H, self.g, self.n
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            m.maskkv_rotate(self.desc, self.rotary, self.prompt_at, self.P, None, None, self.K, self.Kfull[:, :, :self.P], stream)
            m.maskkv_score(self.prompt, self.Qm, self.Kfull, 0.0, self.scores, self.P, None, self.ws[0], stream)
            m.maskkv_select(self.prompt, self.scores, self.P, 1, m.POOL_MEAN, self.budgets, self.idx, self.cu, self.cap, self.ws[1], stream)
            m.maskkv_compact(self.prompt, self.Kfull, self.V_, self.idx, self.cu, self.cap, self.Kc, self.Vc, stream)
            for s in self.step:
                m.maskkv_tree_mask(s["parents"], s["mask"], stream)
                m.maskkv_rotate(self.desc, self.rotary, s["at"], n, s["Q"], s["Qr"], s["K"], s["Kr"], stream)
                m.maskkv_attend_tree(self.desc, s["Qr"], self.Kc, self.Vc, self.cu, self.cap, s["Kr"], s["V"], s["mask"], 0.0, s["O"], s["lse"], self.ws[2], stream)
                s["logits"].copy_(s["O"].transpose(1, 2).reshape(B * n, -1).float().mul(8.0).index_select(1, self.cols))
                m.maskkv_sample(s["logits"], *self.given, s["u"], s["token"], s["prob"], s["logprob"], self.ws[3], stream)

    def outputs(self):
        return [self.Kfull, self.idx, self.cu, self.Kc, self.Vc] + [s[k] for s in self.step for k in ("mask", "Qr", "Kr", "O", "lse", "token", "prob", "logprob")]

    def check(self):
        """Every call against its definition, on what the one before has left."""
        torch.cuda.synchronize()
        f64 = lambda t: t.double().cpu().numpy()
        freq, amplitude = do.frequencies(self.d, 10000.0, "bands", 2.0, 512.0)
        half = mh.HALF[self.dtype]

        def rotated(got, x, at):
            want = do.rotate(x, at, freq, amplitude, self.d, "halves")
            # (10 u of two elements' magnitudes, see test_gpu_rotate.py; then a rounding)
            assert np.all(np.abs(got - want) <= amplitude * 2 * np.abs(x).max() * 12 * mh.U + np.abs(want) * half * 1.02)

        K = f64(self.Kfull)[:, :, :self.P]
        for b in range(self.B):
            rotated(K[b], self.k[b], np.arange(self.P))
        idx, cu = self.idx.cpu().numpy(), self.cu.cpu().numpy()
        scores = self.scores.cpu().numpy()
        Kc, Vc = f64(self.Kc), f64(self.Vc)
        for i in range(self.B * self.H):
            keep = idx[cu[i]:cu[i + 1]]
            assert np.array_equal(keep, orc.select(scores[i], len(keep)))
            assert np.array_equal(Kc[cu[i]:cu[i + 1]], K[i // self.H, i % self.H, keep])
        for j, s in enumerate(self.step):
            q, k, v = self.rows[j]
            Qr, Kr, O, lse = f64(s["Qr"]), f64(s["Kr"]), f64(s["O"]), f64(s["lse"]).reshape(self.B * self.H, self.g, self.n)
            mask = s["mask"].cpu().numpy().view(np.uint32)
            for b in range(self.B):
                rotated(Qr[b], q[b], self.at[j, b])
                rotated(Kr[b], k[b], self.at[j, b])
                sees = do.tree(self.parents[j, b])
                assert np.array_equal(mask[b], do.words(sees))
                for h in range(self.H):
                    i = b * self.H + h
                    heads = slice(h * self.g, (h + 1) * self.g)
                    want, norm, mass = do.attend(Qr[b, heads], Kc[cu[i]:cu[i + 1]], Vc[cu[i]:cu[i + 1]], Kr[b, h], v[b, h], sees)
                    e = mh.logit_error(Qr[b, heads].reshape(-1, self.d), np.concatenate((Kc[cu[i]:cu[i + 1]], Kr[b, h])), 1.0 / np.sqrt(self.d), norm)
                    keys = cu[i + 1] - cu[i] + self.n
                    assert np.all(np.abs(O[b, heads] - want) <= mass * (2 * e + 2 * (keys + 40) * mh.U + half * 1.02) + np.abs(want) * half * 1.02 + 1e-30)
                    assert np.all(np.abs(lse[i] - norm) <= 2 * e + (keys + 40) * mh.U)
            logits, token, prob = f64(s["logits"]), s["token"].cpu().numpy(), f64(s["prob"])
            T, top_k, top_p, min_p = (np.float32(self.limits[0]), self.limits[1], np.float32(self.limits[2]), np.float32(self.limits[3]))
            for r in range(self.B * self.n):
                want, p, _, margin = do.sample(logits[r], T, top_k, top_p, min_p, self.u[j, r])
                assert margin < 1e-10 or (token[r] == want and abs(prob[r] - p) <= 1.02 * mh.U * p + 1e-12)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("kw", [dict(), dict(dtype="f32", g=1, n=5), dict(d=128, g=7, H=1, n=40, keep=500), dict(B=1, n=1, V=50)])
def test_a_program_against_the_definitions(kw):
    if kw.get("n") == 1:
        p = Program(1, **kw)
        p.parents[:] = -1
        for j, s in enumerate(p.step):
            s["parents"].fill_(-1)
    else:
        p = Program(1, **kw)
    p.run()
    p.check()


@pytest.mark.parametrize("kw", [dict(), dict(d=128, g=7, H=1, n=40, keep=500)])
def test_graph_replays_match_the_eager_calls(kw):
    p = Program(2, **kw)
    p.run()
    torch.cuda.synchronize()
    want = [x.clone() for x in p.outputs()]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        p.run()
    for _ in range(3):
        for x in p.outputs():
            x[...] = 0
        p.Kfull[:, :, p.P:] = want[0][:, :, p.P:]
        for w in p.ws:
            if w is not None:
                w.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(p.outputs(), want)


def test_two_programs_on_two_streams():
    a, b = Program(3), Program(4, d=128, g=7, H=1, n=40, keep=500)
    for p in (a, b):
        p.run()
    torch.cuda.synchronize()
    want = [[x.clone() for x in p.outputs()] for p in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for p, s in zip((a, b), streams):
            p.run(s)
    torch.cuda.synchronize()
    for p, w in zip((a, b), want):
        assert same(p.outputs(), w)


def test_the_attention_of_a_tree_feeds_accumulate():
    """The normalisers of maskkv_attend_tree are what maskkv_accumulate takes: a cached row's weights, summed over the rows, and what the rows give to each
    other add up to one for each row."""
    p = Program(5, n=20)
    p.run()
    s = p.step[0]
    w = torch.zeros(p.cap, dtype=torch.float32, device="cuda")
    p.m.maskkv_accumulate(p.desc, s["Qr"], p.Kc, p.cu, p.cap, 0.0, s["lse"], 0.0, None, w)
    torch.cuda.synchronize()
    w, cu = w.double().cpu().numpy(), p.cu.cpu().numpy()
    lse = s["lse"].double().cpu().numpy().reshape(p.B * p.H, p.g, p.n)
    Qr, Kr = s["Qr"].double().cpu().numpy(), s["Kr"].double().cpu().numpy()
    for i in range(p.B * p.H):
        b, h = i // p.H, i % p.H
        sees = do.tree(p.parents[0, b])
        among = np.exp(Qr[b, h * p.g:(h + 1) * p.g] @ Kr[b, h].T / np.sqrt(p.d) - lse[i][..., None]) * sees
        # (normalisers and logits are off by about 1e-5 at most, each of g * n rows)
        assert abs(w[cu[i]:cu[i + 1]].sum() + among.sum() - p.g * p.n) <= 5e-5 * p.g * p.n
