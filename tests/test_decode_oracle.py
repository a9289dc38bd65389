"""The definitions of rotary positions, masks and draws against brute force (CPU)."""
import math

import numpy as np
import pytest

from oracle import decode_oracle as do


def test_a_rotation_keeps_lengths_and_depends_on_distances_only():
    rng = np.random.default_rng(0)
    freq, amplitude = do.frequencies(16, 10000.0)
    assert amplitude == 1.0 and freq[0] == 1.0 and np.isclose(freq[-1], 10000.0 ** (-14 / 16))
    q, k = rng.standard_normal((2, 1, 20))
    for layout in ("halves", "pairs"):
        at = lambda x, p: do.rotate(x, [p], freq, 1.0, 16, layout)[0]
        assert np.isclose(np.linalg.norm(at(q, 12345)), np.linalg.norm(q))
        assert np.isclose(at(q, 700) @ at(k, 655), at(q, 45) @ at(k, 0))
        assert np.array_equal(at(q, 9)[16:], q[0, 16:])
        assert np.allclose(do.rotate(do.rotate(q, [31], freq, 1.0, 16, layout), [-31], freq, 1.0, 16, layout), q)
    quarter = do.rotate(np.array([[1.0, 0.0]]), [1], [math.pi / 2], 2.0, 2, "pairs")
    assert np.allclose(quarter, [[0.0, 2.0]])


def test_scaled_frequencies():
    plain, _ = do.frequencies(64, 500000.0)
    linear, _ = do.frequencies(64, 500000.0, "linear", 4.0)
    assert np.allclose(linear * 4.0, plain)
    based, _ = do.frequencies(64, 500000.0, "base", 4.0)
    assert based[0] == plain[0] and np.isclose(based[-1], plain[-1] / 4.0)
    bands, amplitude = do.frequencies(64, 500000.0, "bands", 4.0, 8192.0, 1.0, 32.0)
    turns = 8192.0 * plain / (2 * math.pi)
    assert np.isclose(amplitude, 1.0 + 0.1 * math.log(4.0))
    assert np.allclose(bands[turns >= 32], plain[turns >= 32]) and np.allclose(bands[turns <= 1] * 4.0, plain[turns <= 1])
    assert np.all(np.diff(bands) < 0)


def test_a_tree_by_paths():
    parents = [-1, 0, 0, 1, -1, 4, 3, -2, 7, 12, 9]
    paths = {0: [0], 1: [0, 1], 2: [0, 2], 3: [0, 1, 3], 4: [4], 5: [4, 5], 6: [0, 1, 3, 6], 7: [], 8: [8], 9: [9], 10: [9, 10]}
    sees = do.tree(parents)
    for i, path in paths.items():
        assert sorted(np.nonzero(sees[i])[0]) == path
    w = do.words(np.ones((1, 40, 40), dtype=bool))
    assert w.shape == (1, 40, 2) and np.all(w[..., 0] == 0xFFFFFFFF) and np.all(w[..., 1] == 0xFF)


def test_attention_without_keys_and_with_all():
    rng = np.random.default_rng(1)
    Q, Kc, Vc, Kr, Vr = (rng.standard_normal(s) for s in ((2, 3, 8), (5, 8), (5, 8), (3, 8), (3, 8)))
    none = np.zeros((3, 3), dtype=bool)
    O, lse, _ = do.attend(Q, Kc[:0], Vc[:0], Kr, Vr, none)
    assert np.all(O == 0) and np.all(lse == -np.inf)
    O, lse, _ = do.attend(Q, Kc, Vc, Kr, Vr, ~none)
    s = Q @ np.concatenate((Kc, Kr)).T / math.sqrt(8)
    p = np.exp(s)
    assert np.allclose(O, p @ np.concatenate((Vc, Vr)) / p.sum(-1, keepdims=True)) and np.allclose(lse, np.log(p.sum(-1)))


@pytest.mark.parametrize("u,token", [(0.0, 0), (0.24, 0), (0.26, 1), (0.49, 1), (0.51, 2), (0.99, 3), (1.0, 3), (-1.0, 0), (float("nan"), 3)])
def test_four_equal_tokens(u, token):
    got = do.sample([2.0] * 4, 0.7, 0, 1.0, 0.0, u)
    assert got[0] == token and np.isclose(got[1], 0.25) and np.isclose(got[2], math.log(0.25))


def test_limits_by_hand():
    l = np.log([0.1, 0.4, 0.05, 0.25, 0.2])
    share = lambda *a: do.sample(l, *a)[:2]
    assert share(1.0, 1, 1.0, 0.0, 0.9)[0] == 1
    assert share(1.0, 2, 1.0, 0.0, 0.9) == (3, pytest.approx(0.25 / 0.65))
    assert share(1.0, 0, 0.7, 0.0, 0.95) == (4, pytest.approx(0.2 / 0.85))       # 0.4, 0.65, then the one that passes 0.7
    assert share(1.0, 0, 0.0, 0.0, 0.95) == (1, 1.0)
    assert share(1.0, 0, 1.0, 0.45, 0.1) == (1, pytest.approx(0.4 / 0.85))        # 0.18 and more
    assert share(1.0, 3, 0.75, 0.0, 0.99) == (3, pytest.approx(0.25 / 0.65))      # 0.85 of the mass is left by top-k: 0.6375 are asked for
    assert share(0.0, 3, 0.75, 0.0, 0.99) == (1, 1.0)
    assert do.sample([np.nan, 1.0, np.inf, np.inf], 1.0, 0, 1.0, 0.0, 0.6)[:3] == (3, 0.5, pytest.approx(math.log(0.5)))
    assert do.sample([-np.inf, np.nan], 1.0, 0, 1.0, 0.0, 0.6)[0] == -1
    assert do.sample([1.0, 1.0, 1.0], 1.0, 2, 1.0, 0.0, 0.6)[0] == 1              # ties: the lower numbers stay


def test_draws_follow_the_distribution():
    rng = np.random.default_rng(2)
    l = rng.standard_normal(6)
    p = np.exp(l / 0.5) / np.exp(l / 0.5).sum()
    us = (np.arange(2000) + 0.5) / 2000
    counts = np.bincount([do.sample(l, 0.5, 0, 1.0, 0.0, u)[0] for u in us], minlength=6)
    assert np.abs(counts / 2000 - p).max() <= 1 / 2000
