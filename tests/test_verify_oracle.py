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


# ---------------------------------------------------------------------------------------------------- exactly
ABOVE = 1.0 - 2.0 ** -24  # the largest random number


def _least_that_fails(holds):
    """How many of the numbers 0, 2^-24, .. below one `holds` of, which falls from true to false: their share of [0, 1), to 2^-24."""
    if not holds(0.0):
        return 0.0
    lo, hi = 0, 1 << 24
    while hi - lo > 1:
        mid = (lo + hi) // 2
        lo, hi = (mid, hi) if holds(mid * 2.0 ** -24) else (lo, mid)
    return hi * 2.0 ** -24


def _outcomes(p, q, tokens, parent, distinct):
    """{(accepted nodes, next token): probability} over all random numbers, by the oracle's own borders: a node's acceptance, given those before it, falls with its
    number, and the next token rises with its."""
    n, V = len(tokens), p.shape[1]
    accept, result = [ABOVE] * n, {}
    call = lambda choose=0.0: tree_verify(p, q, tokens, parent, n, accept, choose, distinct)  # noqa: E731

    def accepted(i, u):
        accept[i] = u
        return i in call()[0]

    def walk(at, i, probability):
        while i < n and parent[i] != at:
            i += 1
        if i == n:
            path = tuple(call()[0])
            assert path[-1] == at
            ends = [0.0] + [_least_that_fails(lambda c, v=v: call(c)[1] <= v) for v in range(V)]
            assert ends[-1] == 1.0
            for v in range(V):
                if ends[v + 1] > ends[v]:
                    result[path, v] = result.get((path, v), 0.0) + probability * (ends[v + 1] - ends[v])
            return
        share = _least_that_fails(lambda u: accepted(i, u))
        if share > 0:
            accept[i] = 0.0
            walk(i, i + 1, probability * share)
        accept[i] = ABOVE
        if share < 1:
            walk(at, i + 1, probability * (1 - share))

    walk(0, 1, 1.0)
    return result


def _drafts(row, kids, drafts):
    """(tokens, probability) of `kids` continuations drawn from `row`."""
    V = len(row)
    for draft in itertools.permutations(range(V), kids) if drafts == "distinct" else itertools.product(range(V), repeat=kids):
        weight, left = 1.0, 1.0
        for x in draft:
            weight *= row[x] / left
            if drafts == "distinct":
                left -= row[x]
        if weight > 0:
            yield draft, weight


def _rows(seed, V, n, filtered=False):
    """n target and draft rows that differ by a good deal; filtered: the target lacks a token."""
    rng = np.random.default_rng(seed)
    p, q = (np.stack([_soft(rng, V) for _ in range(n)]) for _ in range(2))
    if filtered:
        p[np.arange(n), rng.integers(0, V, n)] = 0.0
        p /= p.sum(-1, keepdims=True)
    return p, q


@pytest.mark.parametrize("seed,filtered", [(0, False), (1, True), (2, False)])
@pytest.mark.parametrize("drafts,kids", [("sampled", 1), ("sampled", 2), ("sampled", 3), ("distinct", 1), ("distinct", 2), ("distinct", 3), ("given", 1), ("given", 2), ("given", 3)])
def test_the_first_token_is_exactly_the_targets(drafts, kids, seed, filtered):
    """Over all drafts and all random numbers.  Every border is known to 2^-24: `kids` of acceptances and two of the choice for each outcome."""
    V = 4
    p, q = _rows(10 * seed + kids, V, kids + 1, filtered)
    given = np.random.default_rng(seed).dirichlet(np.ones(V))
    got = np.zeros(V)
    for draft, weight in _drafts(given if drafts == "given" else q[0], kids, drafts):
        for (path, token), share in _outcomes(p, None if drafts == "given" else q, [0, *draft], [-1] + [0] * kids, drafts == "distinct").items():
            got[draft[path[1] - 1] if len(path) > 1 else token] += weight * share
    assert np.abs(got - p[0]).max() <= (kids + 2) * 2.0 ** -24


@pytest.mark.parametrize("above", [1, 2])
@pytest.mark.parametrize("drafts", ["sampled", "distinct", "given"])
def test_the_first_two_tokens_are_exactly_the_targets(drafts, above):
    """A tree of two levels, the second below the first continuation or the other: what a rejection at one node has left means nothing at the next."""
    V = 3
    p, q = _rows(31, V, V + 1)  # row x + 1: behind token x
    parent, got = [-1, 0, 0, above, above], np.zeros((V, V))
    want = p[0][:, None] * p[1:]
    for first, weight in _drafts(q[0], 2, drafts):
        for second, weight2 in _drafts(q[first[above - 1] + 1], 2, drafts):
            rows = [0, first[0] + 1, first[1] + 1, second[0] + 1, second[1] + 1]
            tokens = [0, *first, *second]
            for (path, token), share in _outcomes(p[rows], None if drafts == "given" else q[rows], tokens, parent, drafts == "distinct").items():
                line = [tokens[i] for i in path[1:]] + [token]
                if len(line) == 1:
                    got[line[0]] += weight * weight2 * share * p[line[0] + 1]
                else:
                    got[line[0], line[1]] += weight * weight2 * share
    assert np.abs(got - want).max() <= 6 * 2.0 ** -24  # two acceptances at either node, two borders
