"""Verification of drafted trees in float64, literally: the target's distribution is formed anew after every rejection, max(p - q, 0) normalised, and
with distinct continuations the draft's, without the token that was tried and normalised.  One request at a time."""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import numpy as np


def tree_verify(p, q, tokens: Sequence[int], parent: Optional[Sequence[int]], n_nodes: int, accept, choose: float, distinct: bool = False,
                max_path: Optional[int] = None) -> Tuple[List[int], int]:
    """p, q [nodes, vocab] (q may be None); the accepted nodes and the next token (-1: none)."""
    if n_nodes == 0:
        return [], -1
    clean = lambda v: np.where(np.asarray(v, dtype=np.float64) > 0, v, 0.0).astype(np.float64)  # noqa: E731
    p = clean(p)
    q = None if q is None else clean(q)
    vocab = p.shape[1]
    path, at, tried = [0], 0, 0
    target = p[at].copy()          # (as it is given: not normalised before the first rejection)
    draft = None if q is None else np.asarray(q[at], dtype=np.float64).copy()
    spent, left = 0.0, 1.0         # what distinct continuations have taken of q; what rejections have left of p, without q
    limit = len(tokens) if max_path is None else max_path
    rejected = False
    i = 1
    while i < n_nodes and len(path) < limit:
        above = (i - 1) if parent is None else int(parent[i])
        x = int(tokens[i])
        if above != at or not 0 <= above < i or not 0 <= x < vocab:
            i += 1
            continue
        u = float(np.float32(accept[i]))
        if q is None:
            good = u * left < target[x]
        else:
            ratio_of = draft[x] if not distinct else (draft[x] / (1.0 - spent) if spent < 1.0 else np.inf)
            good = spent < 1.0 and u * ratio_of < target[x]
        if good:
            path.append(i)
            at, target, rejected, spent, left = i, p[i].copy(), False, 0.0, 1.0
            draft = None if q is None else np.asarray(q[i], dtype=np.float64).copy()
        elif q is None:
            left -= target[x]
            target[x] = 0.0
            rejected = True
        elif spent < 1.0:
            now = draft / (1.0 - spent)
            if distinct:
                now = np.where(np.isin(np.arange(vocab), _earlier(tokens, parent, at, i)), 0.0, now)
            rest = clean(target - now)
            total = rest.sum()
            target = rest / total if total > 0 else rest
            rejected = True
            if distinct:
                spent += draft[x]
        i += 1
    weights = clean(target)
    if not weights.sum() > 0:
        weights = clean(p[at])
    total = weights.sum()
    if not total > 0:
        return path, -1
    sums = np.cumsum(weights)
    above = np.flatnonzero(sums > float(np.float32(choose)) * sums[-1])
    return path, int(above[0]) if len(above) else int(np.flatnonzero(weights > 0)[-1])


def _earlier(tokens, parent, at, i):
    """Tokens of the continuations of `at` before node i."""
    return [int(tokens[j]) for j in range(1, i) if ((j - 1) if parent is None else int(parent[j])) == at]
