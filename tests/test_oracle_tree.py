"""The drafted-token oracle against independent facts: torch's softmax attention, rotation as a product
of complex numbers, and the distribution that verification emits."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as O


def test_lines_of_trees_and_chains():
    assert O.lines(None, 3) == [[0], [0, 1], [0, 1, 2]]
    assert O.lines([-1, 0, 0, 1, -2, 4, 9, -1], 8) == [[0], [0, 1], [0, 2], [0, 1, 3], None, None, None, [7]]
    assert O.lines([-1, 0, 1], 3, room=2) == [[0], [0, 1], None]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_is_a_complex_product(layout):
    rng = np.random.default_rng(1)
    x, f = rng.standard_normal(64), O.frequencies(48, 10000.0)
    y = O.rotate(x, 777, layout, 48, f, 1.1)
    a, b = (slice(0, 24), slice(24, 48)) if layout == "half" else (slice(0, 48, 2), slice(1, 48, 2))
    z = (x[a] + 1j * x[b]) * 1.1 * np.exp(1j * 777 * np.array(f))
    np.testing.assert_allclose(y[a] + 1j * y[b], z, rtol=1e-12)
    np.testing.assert_array_equal(y[48:], x[48:])


def test_scaled_frequencies():
    f = O.frequencies(128, 500000.0)
    assert f[0] == 1.0 and f[-1] < 1e-5
    w = O.frequencies(128, 500000.0, "wavelength", 8.0, 1.0, 4.0, 8192)
    assert w[0] == f[0] and math.isclose(w[-1], f[-1] / 8)
    i = O.frequencies(128, 500000.0, "index", 16.0, 1.0, 32.0, 8192)
    assert i[0] == f[0] and math.isclose(i[-1], f[-1] / 16)
    assert all(a >= b for a, b in zip(w, w[1:])) and all(a >= b for a, b in zip(i, i[1:]))
    assert O.frequencies(128, 500000.0, "linear", 4.0)[3] == f[3] / 4


def test_attention_matches_torch():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal(16), rng.standard_normal((9, 16)), rng.standard_normal((9, 16))
    seen = [0, 2, 3, 8]
    want = torch.softmax(torch.tensor(k[seen] @ q * 0.25), 0) @ torch.tensor(v[seen])
    np.testing.assert_allclose(O.attention(q, k, v, seen, 0.25)[0], want.numpy(), rtol=1e-12)
    assert not O.attention(q, k, v, [], 0.25)[0].any()


@pytest.mark.parametrize("form", ["tree", "twins", "draft"])
def test_verification_emits_the_targets_distribution(form):
    """The first emitted token over a fine grid of random numbers has the target's probabilities at node 0."""
    rng = np.random.default_rng(3)
    V, n = 5, 40
    logits = rng.standard_normal((3, V))
    p = O.softmax(logits[0], 0.8)
    draft = rng.standard_normal((2, V)) if form == "draft" else None
    q = O.softmax(draft[0], 0.8) if form == "draft" else None
    grid = (np.arange(n) + 0.5) / n
    got = np.zeros(V)
    # node 0's children: 1 and 2 (trees) or 1 (chain); a drafted token follows q, or is fixed
    for x in range(V) if form == "draft" else [2]:
        tokens = [0, x, 2 if form == "twins" else 4]
        for u0 in grid:
            for u1 in grid:
                for u2 in grid[::4] if form == "tree" else [0.5]:
                    ids, _ = O.verify(logits, tokens, [u0, u1, u2], None if form == "draft" else [-1, 0, 0], draft, 0.8)
                    got[ids[0]] += (q[x] if form == "draft" else 1.0)
    got /= got.sum()
    # a grid of n points places each border within 1 / n (n / 4 points: 4 / n), and at most three meet
    np.testing.assert_allclose(got, p, atol=(4 if form == "tree" else 2) / n)


def test_verification_greedy_and_degenerate_rows():
    logits = np.array([[0.0, 3.0, 3.0], [5.0, 1.0, 1.0], [np.nan, -np.inf, -np.inf]])
    assert O.verify(logits, [0, 1, 0], None, None, None, 0.0) == ([1, 0, -1], [0, 1, 2])
    assert O.verify(logits, [0, 2, 0], None, None, None, 0.0) == ([1], [0])
    assert O.verify(logits[2:], [0], [0.5])[0] == [-1]
    assert O.verify(np.array([[1.0, np.inf, np.inf]]), [0], [0.6])[0] == [2]
