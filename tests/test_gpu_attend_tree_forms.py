"""Every form that maskkv_attend_tree may take (tests/test_attend_tree_plan.py names them and asserts that the plan is the form that a case is here for): who sees whom,
infinities and NaN, captured and replayed (needs an MI355X).  The bound is that of the other tests of this call."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from tests import mx_helpers as mh
from tests.test_attend_tree_plan import FORMS, plan_of
from tests.test_gpu_attend_tree import Case

pytestmark = pytest.mark.gpu

U = mh.U


def case(name, seed, sees):
    dtype, B, H, g, d, n, lens, tile_rows, dealt, shared = FORMS[name]
    p = plan_of(name)
    assert (p.tile_rows, p.chunk > 0, bool(p.shared)) == (tile_rows, dealt, shared), p
    return Case(seed, B, H, d, n, lens, g=g, dtype=dtype, sees=sees)


def some_heads(c):
    """The longest ones, an empty one and the last one."""
    order = np.argsort(c.lens)
    return sorted({int(order[-1]), int(order[len(order) // 2]), int(order[0]), c.B * c.H - 1})


def reference(q, k, v, kr, vr, sees):
    """The definition with all query rows at once: outputs, normalisers and sum_j a_ij |v_j| of finite values; a value that is not finite counts for the rows that
    see it only."""
    g, n, d = q.shape
    keys, values = np.concatenate((k, kr)).astype(np.float64), np.concatenate((v, vr)).astype(np.float64)
    who = np.concatenate((np.ones((n, len(k)), dtype=bool), sees), axis=1)
    O, lse, mass = np.zeros((g, n, d)), np.full((g, n), -np.inf), np.zeros((g, n, d))
    finite = np.isfinite(values)
    with np.errstate(invalid="ignore", over="ignore"):
        for h in range(g):
            s = np.where(who, q[h].astype(np.float64) @ keys.T / np.sqrt(d), -np.inf)
            top = s.max(axis=1, keepdims=True)
            p = np.where(who, np.exp(s - np.where(np.isneginf(top), 0.0, top)), 0.0)
            total = p.sum(axis=1, keepdims=True)
            a = p / np.where(total == 0, 1.0, total)
            O[h], mass[h] = a @ np.where(finite, values, 0.0), a @ np.abs(np.where(finite, values, 0.0))
            for j in np.nonzero(~finite.all(axis=1))[0]:
                O[h] += np.where(who[:, j:j + 1] & ~finite[j], a[:, j:j + 1] * values[j], 0.0)
            lse[h] = np.where(total == 0, -np.inf, top + np.log(np.where(total == 0, 1.0, total)))[:, 0]
    return O, lse, mass


def check(c, heads):
    torch.cuda.synchronize()
    O, lse = c.O.double().cpu().numpy(), c.lse.double().cpu().numpy().reshape(c.B * c.H, c.g, c.n)
    half = mh.HALF[c.dtype]
    for i in heads:
        b, h = i // c.H, i % c.H
        a, z = c.cu[i], c.cu[i + 1]
        q = c.q[b, h * c.g:(h + 1) * c.g]
        want, norm, mass = reference(q, c.k[a:z], c.v[a:z], c.kr[b, h], c.vr[b, h], c.sees[b])
        got, gl = O[b, h * c.g:(h + 1) * c.g], lse[i]
        nothing = norm == -np.inf
        assert np.all(got[nothing] == 0.0) and np.all(gl[nothing] == -np.inf), f"head {i}: rows that see nothing"
        assert np.array_equal(np.isnan(gl), np.isnan(norm)) and np.array_equal(np.isnan(got), np.isnan(want)), f"head {i}: NaN"
        some = np.isfinite(norm)
        if not some.any():
            continue
        assert np.array_equal(np.isinf(got[some]), np.isinf(want[some])) and np.all((got == want)[some][np.isinf(want[some])]), f"head {i}: infinities"
        keys = np.nan_to_num(np.concatenate((c.k[a:z], c.kr[b, h])), posinf=0, neginf=0)
        e = mh.logit_error(q.reshape(-1, c.d), keys, 1.0 / np.sqrt(c.d), norm[some])
        m = len(keys)
        bound = mass * (2 * e + 2 * (m + 40) * U + half * 1.02) + np.abs(want) * half * 1.02 + 1e-30
        ordinary = some[..., None] & np.isfinite(want)
        off = (np.abs(got[ordinary] - want[ordinary]) / bound[ordinary]).max() if ordinary.any() else 0.0
        assert off <= 1.0, f"head {i}: an output is {off:.2f} times its bound off"
        assert np.abs(gl[some] - norm[some]).max() <= 2 * e + (m + 40) * U, f"head {i}: a normaliser"


def test_the_reference_is_the_oracle():
    rng = np.random.default_rng(0)
    q, k, v, kr, vr = (rng.standard_normal(s) for s in ((2, 9, 16), (7, 16), (7, 16), (9, 16), (9, 16)))
    sees = rng.random((9, 9)) < 0.4
    sees[4] = False
    kr[2], vr[2], vr[5, ::2], v[3, 1] = np.nan, np.inf, -np.inf, np.inf
    for rows in (k, k[:0]):
        for got, want in zip(reference(q, rows, v[:len(rows)], kr, vr, sees)[:2], do.attend(q, rows, v[:len(rows)], kr, vr, sees)[:2]):
            assert np.allclose(got, want, rtol=1e-12, atol=1e-12, equal_nan=True)


@pytest.mark.parametrize("sees", ["tree", "any", "none"])
@pytest.mark.parametrize("name", FORMS)
def test_forms(name, sees):
    c = case(name, 40, sees)
    c.run()
    check(c, some_heads(c))


@pytest.mark.parametrize("name", FORMS)
def test_infinities_and_nan(name):
    """In what no row sees, and in what one row sees: at both ends of the response, at the last and first place of a tile, and in the last cached row of the longest head."""
    c = case(name, 41, "any")
    n = c.n
    bad = sorted({j for j in (0, n // 2, 31, 32, 63, 64, n - 1) if j < n})
    for j, x in zip(bad, (np.nan, np.inf, -np.inf, np.nan, np.inf, -np.inf, np.nan)):
        c.sees[:, :, j] = False
        c.kr[:, :, j], c.vr[:, :, j] = x, x
    heads = some_heads(c)
    c.upload()
    c.run()
    check(c, heads)
    assert bool(torch.isfinite(c.O).all())
    c.sees[:, n // 3, bad[0]] = True                              # one row sees a NaN
    c.upload()
    c.run()
    check(c, heads)
    c.kr = np.nan_to_num(c.kr, nan=0.5, posinf=0.5, neginf=0.5)   # and infinite values with finite logits
    c.sees[:, n // 3, bad[0]] = False
    c.sees[:, n // 4, bad[len(bad) // 2]] = True
    for j in bad:
        c.vr[:, :, j] = np.where(np.arange(c.d) % 2, np.inf, -np.inf)
    longest = int(np.argmax(c.lens))
    c.v[c.cu[longest + 1] - 1, ::3] = np.inf
    c.upload()
    c.run()
    check(c, heads)


@pytest.mark.parametrize("name", FORMS)
def test_captured_replayed_and_equal_bits(name):
    c = case(name, 42, "blocks").run()
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
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.O, want[0])


@pytest.mark.parametrize("name", [x for x in FORMS if "128 rows" in x])
def test_strides_of_the_wide_kernel(name):
    """A token's heads together, and rows apart from each other with NaN between them."""
    c = case(name, 43, "blocks").run()
    torch.cuda.synchronize()
    want = (c.O.clone(), c.lse.clone())
    for name in ("Q", "Kr", "Vr", "O"):
        t = getattr(c, name)
        setattr(c, name, t.transpose(1, 2).contiguous().transpose(1, 2))
    c.O.zero_()
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.O, want[0]) and torch.equal(c.lse, want[1])
    for name in ("Q", "Kr", "Vr", "O"):
        t = getattr(c, name)
        w = torch.full((t.shape[0], t.shape[1], t.shape[2] + 70, t.shape[3] + 8), float("nan"), dtype=t.dtype, device="cuda")
        w[:, :, :t.shape[2], :t.shape[3]] = t
        setattr(c, name, w[:, :, :t.shape[2], :t.shape[3]])
    c.O.zero_()
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.O, want[0]) and torch.equal(c.lse, want[1])
    assert bool(torch.isnan(c.O._base[:, :, c.n:]).all() and torch.isnan(c.O._base[..., c.d:]).all())
