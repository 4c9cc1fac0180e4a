"""The oracle of drafted trees against the oracle of block steps, by brute force and by hand (no GPU)."""
import math

import numpy as np
import pytest

from oracle import roco_oracle as orc
from oracle import trees


def _state(rng, n, B, d):
    st = orc.CacheState(np.zeros((B, d)), np.zeros((B, d)), np.zeros(B), np.zeros(B), np.zeros(B), np.full(B, -1, dtype=np.int64), n)
    st.K[:n], st.V[:n] = rng.standard_normal((n, d)), rng.standard_normal((n, d))
    st.count[:n] = rng.integers(1, 50, n)
    mean = np.exp(rng.standard_normal(n)) / B
    st.acc[:n] = np.float32(mean * st.count[:n])
    st.acc2[:n] = np.float32((mean ** 2 * (1 + np.exp(rng.standard_normal(n)))) * st.count[:n])
    st.pos[:n] = rng.permutation(n)
    return st


def _copy(st):
    return orc.CacheState(st.K.copy(), st.V.copy(), st.acc.copy(), st.acc2.copy(), st.count.copy(), st.pos.copy(), st.n_used)


@pytest.mark.parametrize("n,B,window", [(0, 12, 0), (5, 12, 0), (8, 12, 3), (3, 40, 0)])
def test_a_chain_that_evicts_nothing_is_a_block(n, B, window):
    rng = np.random.default_rng(n + B)
    d, b, sc = 8, 4, 1 / math.sqrt(8)
    st = _state(rng, n, B, d)
    q, k, v = (rng.standard_normal((b, d)) for _ in range(3))
    want = _copy(st)
    block = orc.encode_block(want, q, k, v, 60, 4, sc, window, 0.5)
    r = trees.tree_attend(st.K[:n], st.V[:n], st.pos, q[:, None], k, v, [-1, 0, 1, 2], 60, sc, window, 0.5)
    np.testing.assert_allclose(r.out[:, 0], block.out, rtol=1e-12, atol=1e-13)
    c = trees.tree_commit(st, B, q[:, None], k, v, r.lse, [0, 1, 2, 3], 60, 4, sc, window, 0.5)
    for name in ("K", "V", "acc", "acc2", "count", "pos"):
        np.testing.assert_allclose(getattr(st, name), getattr(want, name), rtol=1e-12, atol=1e-13, err_msg=name)
    assert st.n_used == want.n_used and list(c.slots) == list(block.slots) and (c.evicted_slot == -1).all()


def test_victims_are_those_of_a_block_step():
    rng = np.random.default_rng(3)
    d, B, sc = 8, 30, 0.4
    for policy in (None, orc.Policy("aas", "all"), orc.Policy("mas", "window"), orc.Policy("oldest", "all", 4)):
        st = _state(rng, B - 2, B, d)
        want = _copy(st)
        q, k, v = (rng.standard_normal((5, d)) for _ in range(3))
        block = orc.encode_block(want, q, k, v, 60, 9, sc, policy=policy)
        c = trees.tree_commit(st, B, q[:, None], k, v, np.zeros((5, 1)), [0, 1, 2, 3, 4], 60, 9, sc, policy=policy)
        assert list(c.slots) == list(block.slots)
        assert list(c.evicted_slot) == list(block.evicted_slot) and list(c.evicted_pos) == list(block.evicted_pos)


def test_nodes_that_a_node_sees():
    sees = trees.seen_nodes([-1, 0, 0, 1, 9, 4, -7], 7)  # 9 is no earlier node: node 4 is a root
    assert [np.flatnonzero(row).tolist() for row in sees] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], [6]]


def test_page_tables_by_hand():
    table, pages, rows, slots = trees.page_tables([0, 17, 5], [3, 33, 5], 16, [7, 2, 9], [[-1, -1, -1], [4, 8, -1], [1, -1, -1]], 25, False)
    assert table.tolist() == [[7, -1, -1], [4, 8, 2], [1, -1, -1]]
    assert pages.tolist() == [0, 1, 2, 2] and rows.tolist() == [0, 3, 19, 19]
    assert slots.tolist() == [112, 113, 114] + [8 * 16 + i for i in range(1, 16)] + [32] + [-1] * 6
