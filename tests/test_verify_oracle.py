"""The oracle of the verification: whatever was drafted, tokens come as the target's probabilities say."""
import itertools

import numpy as np
import pytest

from oracle.verify import tree_verify


def _soft(rng, *shape):
    x = np.exp(rng.standard_normal(shape) * 1.5)
    return x / x.sum(-1, keepdims=True)


@pytest.mark.parametrize("drafts,kids", [("sampled", 1), ("sampled", 3), ("distinct", 1), ("distinct", 2), ("distinct", 3), ("given", 2)])
def test_the_first_token_is_the_targets(drafts, kids):
    """Over all drafts, with their probabilities, and the exact shares of the random numbers' ranges by quadrature over a fine grid of midpoints."""
    rng = np.random.default_rng(kids)
    V = 4
    p = np.stack([_soft(rng, V) for _ in range(kids + 1)])
    q = np.stack([_soft(rng, V) for _ in range(kids + 1)])
    got = np.zeros(V)
    parent = [-1] + [0] * kids
    n, n_choose = (400, 64) if kids == 1 else (20, 20) if kids == 2 else (7, 6)
    grid, choices = (np.arange(n) + 0.5) / n, (np.arange(n_choose) + 0.5) / n_choose
    orders = itertools.product(range(V), repeat=kids) if drafts != "distinct" else itertools.permutations(range(V), kids)
    given = _soft(rng, V)
    for draft in orders:
        weight, left = 1.0, 1.0
        for x in draft:
            weight *= given[x] if drafts == "given" else q[0, x] / left
            if drafts == "distinct":
                left -= q[0, x]
        for u in itertools.product(grid, repeat=kids):
            path = None
            # (whatever is chosen at the end, the path is the same)
            for c in choices:
                path, token = tree_verify(p, None if drafts == "given" else q, [0, *draft], parent, kids + 1, [0.0, *u], c, drafts == "distinct")
                first = draft[path[1] - 1] if len(path) > 1 else token
                if len(path) > 1:
                    got[first] += weight / n ** kids
                    break
                got[first] += weight / n ** kids / n_choose
    # midpoints: each range's share is off by at most one cell of either grid (kids of the one, one of the other, for every token's border)
    assert np.abs(got - p[0]).max() <= kids / n + 1.0 / n_choose
    assert abs(got.sum() - 1) < 1e-9


def test_a_chain_is_a_tree():
    rng = np.random.default_rng(9)
    for _ in range(50):
        p, q = _soft(rng, 5, 7), _soft(rng, 5, 7)
        tokens, accept, choose = rng.integers(0, 7, 5), rng.random(5), rng.random()
        assert tree_verify(p, q, tokens, None, 5, accept, choose) == tree_verify(p, q, tokens, [-1, 0, 1, 2, 3], 5, accept, choose)


def test_sizes_and_what_counts_as_zero():
    p, q = np.array([[0.5, np.nan, 0.5, -1.0]] * 2), np.array([[0.25] * 4] * 2)
    assert tree_verify(p, q, [0, 1], None, 0, [0, 0], 0.0) == ([], -1)
    assert tree_verify(p, q, [0, 1], None, 2, [0, 0], 0.0) == ([0], 0)      # token 1 has no probability
    assert tree_verify(p, q, [0, 2], None, 2, [0, 0.9], 0.99) == ([0, 1], 2)
    assert tree_verify(p, q, [0, 2], None, 2, [0, 0.9], 0.99, max_path=1) == ([0], 2)
    assert tree_verify(-p, q, [0, 2], None, 1, [0, 0], 0.5) == ([0], 3)
    assert tree_verify(np.zeros((2, 4)), q, [0, 2], None, 2, [0, 0], 0.5) == ([0], -1)
