"""Pins of the drafted-token oracle: what the definitions promise, on cases small enough to work out."""
import itertools

import numpy as np
import pytest

from oracle import draft_oracle as orc


def test_tree_rows():
    seen, depth = orc.tree_rows([-1, 0, 0, 2, 1, -1, 5, 9])
    assert seen == [{0}, {0, 1}, {0, 2}, {0, 2, 3}, {0, 1, 4}, {5}, {5, 6}, {7}]
    assert depth == [0, 1, 1, 2, 2, 0, 1, 0]
    words = orc.mask_words(orc.tree_rows(list(range(-1, 39)))[0], 2)
    assert words[39].tolist() == [0xFFFFFFFF, 0xFF] and words[31].tolist() == [0xFFFFFFFF, 0] and words[32].tolist() == [0xFFFFFFFF, 1]


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation(interleaved):
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(2, 64))
    f = 100.0 ** (-2.0 * np.arange(16) / 32)
    dot = lambda a, b: float(orc.rotate(q, a, f, 32, interleaved)[0] @ orc.rotate(k, b, f, 32, interleaved)[0])
    assert abs(dot(7, 3) - dot(104, 100)) < 1e-9                      # the distance alone counts
    r = orc.rotate(q, 5, f, 32, interleaved)[0]
    assert np.array_equal(r[32:], q[32:]) and abs(np.linalg.norm(r) - np.linalg.norm(q)) < 1e-12
    assert np.array_equal(orc.rotate(q, 0, f, 32, interleaved)[0], q)
    e = np.zeros(64)
    e[0] = 1.0
    r = orc.rotate(e, 1, f, 32, interleaved, amplitude=2.0)[0]
    assert abs(r[0] - 2 * np.cos(1.0)) < 1e-15 and abs(r[1 if interleaved else 16] - 2 * np.sin(1.0)) < 1e-15


@pytest.mark.parametrize("children", [1, 2, 3])
@pytest.mark.parametrize("drawn", [True, False])
def test_tokens_are_distributed_as_the_target(drawn, children):
    """The first token behind the cache, over a fine grid of all random numbers: its distribution is the target's, whatever
    the drafts' is.  Drawn drafts: every draw weighed with its probability; chosen ones: distinct tokens in any order."""
    p, q = np.array([0.5, 0.2, 0.3]), np.array([0.1, 0.6, 0.3])
    grid = (np.arange(40) + 0.5) / 40
    got = np.zeros(3)
    draws = list(itertools.product(range(3), repeat=children)) if drawn else [tuple(range(2, 2 - children, -1))]
    for tokens in draws:
        weight = np.prod([q[t] for t in tokens]) if drawn else 1.0
        rows = np.tile(p, (1 + children, 1))
        # the outcome depends on the grid point of the first accepted child only: walk the tree of acceptances exactly
        alive, P, left = 1.0, p.copy(), 1.0
        for t in tokens:
            accept = min(1.0, P[t] / q[t]) if drawn else min(1.0, P[t])
            got[t] += weight * alive * accept
            alive *= 1.0 - accept
            rest = np.maximum(P - q, 0) if drawn else np.where(np.arange(3) == t, 0, P)
            P = rest / rest.sum() if rest.sum() > 0 else P
        got += weight * alive * P
        for u in itertools.product(grid[::13], repeat=children):
            kept, nxt = orc.verify([-1] + [0] * children, [0] + list(tokens), rows, np.tile(q, (1 + children, 1)) if drawn else None,
                                   [0.0] + list(u), 0.37)
            P, left, where = p.copy(), 1.0, None
            for i, t in enumerate(tokens):
                if (u[i] * q[t] < P[t]) if drawn else (u[i] < P[t]):
                    where = i
                    break
                rest = np.maximum(P - q, 0) if drawn else np.where(np.arange(3) == t, 0, P)
                P = rest / rest.sum()
            assert kept == ([0] if where is None else [0, where + 1])
            want = p if where is not None else P
            assert nxt == int(np.nonzero(np.cumsum(want) > 0.37 * want.sum())[0][0])
    assert np.allclose(got, p, atol=1e-12)


def test_walk_of_a_tree():
    n = 4
    one = lambda x: np.eye(n)[x]
    target = np.stack([one(2), one(0), one(1), one(3), one(0)])
    parent, token = [-1, 0, 0, 2, 3], [9, 1, 2, 1, 3]
    half = [0.5] * 5
    assert orc.verify(parent, token, target, None, half, 0.5) == ([0, 2, 3, 4], 0)
    assert orc.verify(parent, [9, 1, 2, 0, 3], target, None, half, 0.5) == ([0, 2], 1)
    assert orc.verify(parent, [9, 1, 7, 1, 3], target, None, half, 0.5) == ([0], 2)          # a token outside the vocabulary
    assert orc.verify([-1], [0], np.zeros((1, n)), None, [0.0], 0.5) == ([0], -1)
