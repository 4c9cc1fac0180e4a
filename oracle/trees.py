"""Drafted trees over a budgeted cache, per unit, in float64: attention of all nodes, and the accepted path taken over.

Ranking keys are formed in float32, one rounded operation after the other, as the library defines them, so that both sides take the
same victims: nothing here has to allow for ties.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np

from .roco_oracle import F64, CacheState, Policy, _recency, _second_statistic, k_smallest


def seen_nodes(parent: Sequence[int], n_nodes: int) -> np.ndarray:
    """[n, n] bool: node i sees node j (itself, or a node above it)."""
    sees = np.zeros((n_nodes, n_nodes), dtype=bool)
    for i in range(n_nodes):
        j = i
        while True:
            sees[i, j] = True
            if not 0 <= parent[j] < j:  # anything but an earlier node is none
                break
            j = parent[j]
    return sees


@dataclass
class TreeResult:
    out: np.ndarray   # [nodes, group, d]
    lse: np.ndarray   # [nodes, group]
    mass: np.ndarray  # [nodes, group, d]: sum of p |v|, what errors of the probabilities are relative to
    logit: float      # largest sum of |q k| times the scale: what errors of the logits are relative to


def tree_attend(K, V, pos, q, k_new, v_new, parent, qpos0: int, scale: float, window: int = 0, bias: float = 0.0) -> TreeResult:
    """K, V [n, d] and pos [n] of the cached tokens; q [nodes, group, d], k_new, v_new [nodes, d]."""
    K, V, q, k_new, v_new = (np.asarray(x, dtype=F64) for x in (K, V, q, k_new, v_new))
    T, G, d = q.shape
    n = K.shape[0]
    sees = seen_nodes(parent, T)
    depth = sees.sum(1) - 1
    out, lse, mass, logit = np.zeros((T, G, d)), np.zeros((T, G)), np.zeros((T, G, d)), 0.0
    for i in range(T):
        nodes = np.flatnonzero(sees[i])
        keys, values = np.concatenate([K, k_new[nodes]]), np.concatenate([V, v_new[nodes]])
        at = np.concatenate([np.asarray(pos[:n], dtype=np.int64), qpos0 + depth[nodes]])
        x = (q[i] @ keys.T) * F64(scale) + _recency(np.array([qpos0 + depth[i]]), at, window, bias)
        m = x.max(1, keepdims=True)
        p = np.exp(x - m)
        total = p.sum(1, keepdims=True)
        p = p / total
        out[i] = p @ values
        mass[i] = p @ np.abs(values)
        lse[i] = (m + np.log(total))[:, 0]
        with np.errstate(invalid="ignore"):
            logit = max(logit, float((np.abs(q[i]) @ np.abs(keys).T).max()) * scale)
    return TreeResult(out, lse, mass, logit)


def choose_evictions(state: CacheState, E: int, scope: int, policy: Optional[Policy]) -> np.ndarray:
    n, policy = state.n_used, policy or Policy()
    f = np.float32
    acc, acc2, count, pos = state.acc[:n].astype(f), state.acc2[:n].astype(f), state.count[:n].astype(f), state.pos[:n]
    if policy.importance == "mas":
        importance = acc / count
    elif policy.importance == "oldest":
        importance = np.where(pos < policy.sinks, np.inf, pos.astype(F64))
    else:
        importance = acc if policy.importance == "aas" else acc2
    if policy.scope_kind == "std":
        mean = acc / count
        key = np.maximum(acc2 / count - mean * mean, f(0))
    else:
        key = pos.astype(F64) if policy.scope_kind == "window" else np.zeros(n)
    if policy.scope_kind == "all":
        scope = n
    inside = k_smallest(key, min(n, scope + E - 1))
    return np.sort(inside[k_smallest(importance[inside], E)])


@dataclass
class CommitResult:
    evicted_slot: np.ndarray
    evicted_pos: np.ndarray
    slots: List[int]
    mass: np.ndarray  # [2, slots]: what was added to Acc and Acc2


def tree_commit(state: CacheState, budget: int, q, k_new, v_new, lse, path: Sequence[int], qpos0: int, scope: int, scale: float,
                window: int = 0, bias: float = 0.0, policy: Optional[Policy] = None) -> CommitResult:
    """In place.  q [nodes, group, d], lse [nodes, group]; `path` the accepted nodes; the state's arrays may be longer than `budget`."""
    a, n = len(path), state.n_used
    added = np.zeros((2, state.K.shape[0]))
    if a == 0:
        return CommitResult(np.zeros(0, np.int64), np.zeros(0, np.int64), [], added)
    n_new = min(budget, n + a)
    E = n + a - n_new
    victims = choose_evictions(state, E, min(scope, budget), policy) if E else np.zeros(0, np.int64)
    slots = [int(j) for j in victims] + list(range(n, n_new))
    was = np.array([j < n for j in slots])
    evicted_slot = np.where(was, slots, -1)
    evicted_pos = np.where(was, state.pos[slots], -1)
    token = np.full(n_new, -1)
    token[slots] = np.arange(a)
    for k, j in enumerate(slots):
        state.K[j], state.V[j] = k_new[path[k]], v_new[path[k]]
        state.pos[j] = qpos0 + k
        state.acc[j] = state.acc2[j] = state.count[j] = 0.0
    state.n_used = n_new
    for k in range(a):
        x = (np.asarray(q[path[k]], dtype=F64) @ state.K[:n_new].T) * F64(scale)
        x = x + _recency(np.array([qpos0 + k]), state.pos[:n_new], window, bias)
        seen = token <= k
        p = np.where(seen, np.exp(x - np.asarray(lse[path[k]], dtype=F64)[:, None]).mean(0), 0.0)
        state.acc[:n_new] += p
        state.acc2[:n_new] = _second_statistic(policy, state.acc2[:n_new], p, seen, n + k + 1)
        state.count[:n_new] += seen
        added[0, :n_new] += p
        added[1, :n_new] += p * p
    return CommitResult(evicted_slot, evicted_pos, slots, added)


def page_tables(held, want, page: int, free_pages, table, rows: int, padded: bool):
    """(table, page_start, row_start, map) by counting, request after request."""
    table = np.array(table)
    R, max_pages = table.shape
    most = max_pages * page
    starts, row_starts, entries, taken = [0], [0], [], 0
    for r in range(R):
        h = min(max(int(held[r]), 0), most)
        w = min(max(int(want[r]), h), most)
        for i in range(-(-h // page), -(-w // page)):
            table[r, i] = free_pages[taken] if taken < len(free_pages) else -1
            taken += 1
        mine = [int(table[r, j // page]) * page + j % page if table[r, j // page] >= 0 else -1 for j in range(h, w)]
        entries.append(mine)
        starts.append(taken)
        row_starts.append(row_starts[-1] + len(mine))
    if padded:
        slots = np.full((R, rows), -1)
        for r, mine in enumerate(entries):
            slots[r, :len(mine[:rows])] = mine[:rows]
    else:
        flat = [e for mine in entries for e in mine][:rows]
        slots = np.array(flat + [-1] * (rows - len(flat)))
    return table, np.array(starts), np.array(row_starts), slots
