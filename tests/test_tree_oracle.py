"""Pins of the oracle of drafted trees (oracle/tree.py): rotations against hand cases and their invariants,
tree attention against causal attention along each token's path, commits against hand cases (CPU)."""
import math

import numpy as np
import pytest

from oracle import paged, tree


def test_rotation_by_hand():
    """A quarter turn a position in the first pair, none in the second."""
    x = np.arange(1.0, 65.0)[None]
    f = np.array([math.pi / 2, 0.0])
    y = tree.rotate(x, np.array([1]), 4, tree.HALVES, f)[0]
    assert np.allclose(y[:4], [-3, 2, 1, 4]) and np.array_equal(y[4:], x[0, 4:])
    y = tree.rotate(x, np.array([1]), 4, tree.PAIRS, f)[0]
    assert np.allclose(y[:4], [-2, 1, 3, 4]) and np.array_equal(y[4:], x[0, 4:])
    y = tree.rotate(x, np.array([-1]), 4, tree.PAIRS, f, scale=2.0)[0]
    assert np.allclose(y[:4], [4, -2, 6, 8]) and np.array_equal(y[4:], x[0, 4:])


@pytest.mark.parametrize("layout", [tree.HALVES, tree.PAIRS])
@pytest.mark.parametrize("dim", [2, 10, 64])
def test_rotated_products_depend_on_the_distance_alone(layout, dim):
    rng = np.random.default_rng(dim)
    f, _ = tree.frequencies(dim, 10000.0)
    q, k = rng.standard_normal((2, 1, 64))
    def dot(p, r):
        return (tree.rotate(q, np.array([p]), dim, layout, f) @ tree.rotate(k, np.array([r]), dim, layout, f).T)[0, 0]
    assert np.isclose(dot(7, 3), dot(104, 100)) and np.isclose(dot(0, 5), dot(-5, 0))
    assert not np.isclose(dot(7, 3), dot(7, 4))


def test_scaled_frequencies():
    f, one = tree.frequencies(64, 10000.0)
    assert f[0] == 1.0 and np.isclose(f[-1], 10000.0 ** (-62 / 64)) and one == 1.0
    assert np.allclose(tree.frequencies(64, 10000.0, tree.LINEAR, 4.0)[0], f / 4)
    b, _ = tree.frequencies(64, 10000.0, tree.BASE, 8.0)
    assert b[0] == 1.0 and np.isclose(b[-1], f[-1] / 8)
    p, scale = tree.frequencies(64, 10000.0, tree.PARTS, 8.0, original=4096.0)
    turns = 4096 * f / (2 * math.pi)
    assert np.allclose(p[turns >= 32], f[turns >= 32]) and np.allclose(p[turns <= 1], f[turns <= 1] / 8)
    assert (np.diff(p) < 0).all() and np.isclose(scale, 1 + 0.1 * math.log(8))


def test_masks_and_depths():
    m = tree.masks([-1, 0, 0, 1, 3, 2], 1)[:, 0].tolist()
    assert m == [0b1, 0b11, 0b101, 0b1011, 0b11011, 0b100101]
    assert tree.depths([-1, 0, 0, 1, 3, 2]).tolist() == [0, 1, 1, 2, 3, 2]
    m = tree.masks([-1] + list(range(99)), 2)
    assert m[63].tolist() == [-1, 0] and m[99].tolist() == [-1, (1 << 36) - 1]


def test_tree_attention_is_causal_attention_along_each_path():
    rng = np.random.default_rng(4)
    parents, past, H = [-1, 0, 0, 2, 1, 3, 2], 70, 2
    n = len(parents)
    pool = rng.standard_normal((6, 2, H, 64, 64))
    table = np.array([[4, 1, -1]])
    q = rng.standard_normal((n, H, 64))
    got = tree.attention(q, pool, [], 0, table, [past + n], [0, n], tree.masks(parents, 1))
    for i in range(n):
        path = [i]
        while parents[path[0]] >= 0:
            path.insert(0, parents[path[0]])
        # the same tokens as a sequence of their own
        own = pool.copy()
        for k, j in enumerate(path):
            own[[5, 2][(past + k) // 64 - 1], :, :, (past + k) % 64] = pool[table[0, (past + j) // 64], :, :, (past + j) % 64]
        own[5, :, :, :past - 64] = pool[1, :, :, :past - 64]
        want = paged.shared_attention(q[i:i + 1], own, [], 0, np.array([[4, 5, 2]]), [past + len(path)], None)
        assert np.allclose(got[i], want[0])


def test_tree_attention_of_rows_that_see_nothing():
    pool, q = np.ones((1, 2, 1, 64, 64)), np.ones((3, 1, 64))
    words = np.array([[0], [2], [0]], dtype=np.int64)
    out = tree.attention(q, pool, [], 0, np.array([[0]]), [2], [0, 2], words)
    assert (out[0] == 0).all() and np.allclose(out[1], 1) and np.isnan(out[2]).all()
    assert (tree.attention(q, pool, [], 0, np.array([[0]]), [1], [0, 2], words)[:2] == 0).all()


def test_accepted_paths_by_hand():
    tokens, parents = [5, 7, 8, 7, 9, 8], [-1, 0, 0, 1, 2, 2]
    assert tree.accept(tokens, parents, [8, 0, 9, 0, 4, 0], 8) == ([0, 2, 4], 4)
    assert tree.accept(tokens, parents, [8, 0, 9, 0, 4, 0], 2) == ([0, 2], 9)
    assert tree.accept(tokens, parents, [3, 0, 9, 0, 4, 0], 8) == ([0], 3)
    assert tree.accept([5, 7, 7], [-1, 0, 0], [7, 1, 2], 8) == ([0, 1], 1)      # the first of two alike
    assert tree.accept([5, -1], [-1, 0], [-1, 3], 8) == ([0], -1)               # no choice matches nothing
    assert tree.accept([5, 6, 6], [-1, 2, 0], [6, 1, 4], 8) == ([0, 2], 4)      # parents come first


def test_commit_by_hand():
    pool = np.zeros((2, 3, 2, 1, 64, 64))
    pool[:, 1, :, 0, 60:] = np.arange(4)[:, None] + 1
    pool[:, 0, :, 0, :2] = np.arange(2)[:, None] + 5                             # tokens 60 .. 65: 1 2 3 4 5 6
    tokens, parents, choices = [5, 7, 8, 7, 9, 8], [-1, 0, 0, 1, 2, 2], [8, 0, 8, 0, 4, 11]
    path, counts, chosen, lens, new = tree.commit(tokens, parents, choices, [0, 6], np.array([[1, 0]]), [66], pool, 4)
    assert path.tolist() == [[0, 2, 5, -1]] and counts.tolist() == [3] and chosen.tolist() == [11] and lens.tolist() == [63]
    assert new[0, 1, 0, 0, 60:, 0].tolist() == [1, 3, 6, 4] and new[1, 0, 1, 0, :2, 9].tolist() == [5, 6]
    path, counts, chosen, lens, new = tree.commit(tokens, parents, choices, [0, 0], np.array([[1, 0]]), [66], pool, 4)
    assert counts.tolist() == [0] and chosen.tolist() == [-1] and lens.tolist() == [66] and np.array_equal(new, pool)
