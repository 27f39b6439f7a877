"""The fp64 oracle of steps with drafted tokens: trees against a walk up their
parents, and verification against what it is for, the target's distribution."""
import numpy as np
import pytest

from oracle import drafts as od


@pytest.mark.parametrize("n,words", [(1, 1), (9, 1), (33, 2), (70, 2)])
def test_tree_against_a_walk(n, words):
    rng = np.random.default_rng(n)
    parents = [int(rng.integers(-2, i + 2)) for i in range(n)]   # some of no earlier token
    pos, seen = od.tree(parents, 100, words)
    for i in range(n):
        if i >= 32 * words:
            assert pos[i] == -1 and not seen[i].any()
            continue
        x, up = i, []
        while 0 <= x:
            up.append(x)
            x = parents[x] if 0 <= parents[x] < x else -1
        assert pos[i] == 100 + len(up) - 1 and sorted(np.flatnonzero(seen[i])) == sorted(up)
    bits = od.words_of(seen, words).view(np.uint32)
    for i in range(n):
        for j in range(min(n, 32 * words)):
            assert bool(bits[i, j // 32] >> (j % 32) & 1) == seen[i, j]


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("parents", [[-1, 0], [-1, 0, 0, 0], [-1, 0, 0, 1, 1]])
def test_tokens_are_distributed_as_the_targets(parents, drawn):
    """The token behind the first one, accepted or drawn, over many random
    numbers: shares within five standard deviations, sqrt(p (1 - p) / N)."""
    rng = np.random.default_rng(len(parents) + drawn)
    vocab, N, n = 4, 20000, len(parents)
    p, q = rng.dirichlet(np.ones(vocab), n), rng.dirichlet(np.ones(vocab), n)
    sure = rng.permutation(vocab)
    seen = np.zeros(vocab)
    for _ in range(N):
        ids, first = [0] * n, 0
        for i in range(1, n):
            ids[i] = int(rng.choice(vocab, p=q[parents[i]])) if drawn else int(sure[i % vocab])
        path, after = od.verify(p, ids, parents, rng.random(n), q if drawn else None)
        seen[ids[path[1]] if len(path) > 1 else after] += 1
    assert (np.abs(seen / N - p[0]) <= 5 * np.sqrt(p[0] * (1 - p[0]) / N)).all(), (seen / N, p[0])


def test_verification_by_hand():
    p = np.array([[0.5, 0.25, 0.25, 0.0], [0.0, 0.0, 0.0, 1.0], [0.25, 0.25, 0.25, 0.25]])
    q = np.array([[0.0, 0.0, 1.0, 0.0]] * 3)
    ids, parents = [9, 2, 2], [-1, 0, 0]
    # accepted: 0.2 * 1 < 0.25; behind it nothing but token 3
    assert od.verify(p, ids, parents, [0.9, 0.2, 0.0], q) == ([0, 1], 3)
    # refused, then again: nothing is left of token 2; of [0.5, 0.25] the draw takes 0 up to two thirds
    assert od.verify(p, ids, parents, [0.6, 0.25, 0.0], q) == ([0], 0)
    assert od.verify(p, ids, parents, [0.7, 0.25, 0.0], q) == ([0], 1)
    # a row of q that drew nothing may hold anything
    assert od.verify(p, ids, parents, [0.9, 0.2, 0.0], np.array([q[0], q[0] * np.nan, q[0] * np.nan])) == ([0, 1], 3)
    # without q: 0.3 >= 0.25 refused, the same id again has no weight
    assert od.verify(p, ids, parents, [0.0, 0.3, 0.0]) == ([0], 0)
    # nothing left at all: the draw is from p itself
    assert od.verify(np.array([[0.0, 0.9]] * 2), [0, 1], [-1, 0], [0.5, 1.0]) == ([0], 1)
    assert od.verify(np.zeros((1, 4)), [0], [-1], [0.5]) == ([0], -1)
    assert od.verify(np.zeros((0, 4)), [], [], []) == ([], -1)


def test_residuals_nest():
    """max(max(p - S q, 0) - T q, 0) = max(p - (S + T) q, 0) for q >= 0, so one
    number says what any number of refusals left."""
    rng = np.random.default_rng(1)
    p, q = rng.dirichlet(np.ones(50)), rng.dirichlet(np.ones(50))
    rest, share, left = p, 0.0, 1.0
    for _ in range(6):
        rest, share = np.maximum(rest - left * q, 0), share + left
        left = rest.sum()
        assert np.allclose(rest, np.maximum(p - share * q, 0), atol=1e-15)
