"""Speculative decoding on budgeted caches, and the pages that hold caches of different budgets: what is measured of the operators
roco_tree_attend, roco_tree_commit, roco_page_tables and roco_page_store, beside their plain forms.

A case is a plain dict; `op` names the operator.  Caches, queries and drafted tokens follow the heavy-hitter recipe of `inputs/`: N(0, 1)
rows, a unit vector u per unit, 4 u added to 2 % of the keys and 2 u to every query.  `own` false: elementary torch operations in 32 bits;
`own` true: the library's calls.
"""
import math
import random

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------------------------- cases
def _tree(op, requests, heads, dtype, head_dim, budget, nodes, group=1, page=0, ragged=False, window=0, scope=64, path=0, name=None):
    """A step of `requests` x `heads` units; page > 0: caches in pages, with a budget of each request's own."""
    c = {"op": op, "requests": requests, "heads": heads, "dtype": dtype, "head_dim": head_dim, "budget": budget, "nodes": nodes,
         "group": group, "page": page, "ragged": ragged, "window": window}
    if op == "commit":
        c.update(scope=scope, path=path)
    if name is not None:
        c["name"] = name
    return c


def _tables(requests, page, most, grow, padded, name=None):
    """Requests of up to `most` slots; grow > 0: they hold slots and take up to `grow` more, 0: they are new."""
    c = {"op": "tables", "requests": requests, "page": page, "most": most, "grow": grow, "padded": padded}
    if name is not None:
        c["name"] = name
    return c


def _store(groups, rows, heads, dtype, head_dim, page, name=None):
    """groups > 0: caches [groups, heads, rows, d] of different fills; 0: `rows` new tokens as a fused projection leaves them."""
    c = {"op": "store", "groups": groups, "rows": rows, "heads": heads, "dtype": dtype, "head_dim": head_dim, "page": page}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a tree of one node: the single token of a tiny fp32 layer, nothing but latency
        _tree("attend", 4, 4, "f32", 64, 500, 1, name="attend_one_token"),
        # 16 drafted tokens on the serving batch: 16 sequences x 32 heads x 2048 slots
        _tree("attend", 16, 32, "bf16", 128, 2048, 16, name="attend_serving"),
        # the largest trees of a grouped model on paged caches of different budgets: 512 query rows per unit
        _tree("attend", 16, 8, "bf16", 128, 4096, 64, group=8, page=64, ragged=True, name="attend_wide_pages"),
        # two long contexts, 8 key/value heads shared by 8 query heads each
        _tree("attend", 2, 8, "bf16", 128, 65536, 8, group=8, page=256, name="attend_long_pages"),
        # full precision, odd sizes, a recency window
        _tree("attend", 12, 5, "f32", 128, 1501, 21, ragged=True, window=64, name="attend_ragged_f32"),
        # up to four accepted tokens of a tiny fp32 layer: latency
        _tree("commit", 4, 4, "f32", 64, 500, 8, path=4, scope=32, name="commit_tiny_f32"),
        # up to six accepted tokens on the serving batch
        _tree("commit", 16, 32, "bf16", 128, 2048, 16, path=6, name="commit_serving"),
        # grouped heads, head_dim 64, paged caches of different budgets
        _tree("commit", 24, 8, "bf16", 64, 4096, 32, group=4, page=64, ragged=True, path=8, name="commit_grouped_pages"),
        # between two decode steps: a few new slots for each of 64 requests
        _tables(64, 64, 2048, 8, False, name="tables_step"),
        # tables and maps of a full batch of new prompts
        _tables(1024, 64, 8192, 0, True, name="tables_prompts"),
        # the tokens of one decode step of 64 sequences, straight from the fused projection
        _store(0, 64, 8, "bf16", 128, 64, name="store_step"),
        # 16 compressed prompts x 32 heads into pages
        _store(16, 2048, 32, "bf16", 128, 64, name="store_prompts"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "commit", "commit", "tables", "store"])
    dtype, d = rng.choice([("bf16", 128), ("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
    e = 2 if dtype == "bf16" else 4
    if op == "tables":
        requests = _log_int(rng, 1, 4096)
        return _tables(requests, rng.choice([16, 32, 64, 128]), _log_int(rng, 16, min(8192, max(64, (8 << 20) // requests))),
                       rng.choice([0, 0, 1, 17, 64]), rng.random() < 0.5)
    if op == "store":
        heads, page = rng.choice([1, 4, 5, 8, 32]), rng.choice([16, 32, 64, 128])
        groups = rng.choice([0, 1, 1, 1]) * _log_int(rng, 1, 32)
        most = (128 << 20) // (max(1, groups) * heads * d * e)
        return _store(groups, _log_int(rng, 1, min(most, 4096 if groups else 16384)), heads, dtype, d, page)
    budget = _log_int(rng, 64, 16384)
    heads = rng.choice([1, 2, 5, 8, 8, 32])
    group = rng.choice([1, 1, 2, 3, 4, 8])
    nodes = _log_int(rng, 1, 64)
    # at most the bytes of the serving batch, and the products of the widest listed trees (fp32: a sixteenth of them)
    most = min((256 << 20) // (2 * budget * heads * d * e), (8 << 30) // (budget * heads * d * nodes * group * (1 if e == 2 else 16)))
    requests = _log_int(rng, 1, max(1, min(64, most)))
    page = rng.choice([0, 0, 16, 64, 128])
    ragged = rng.random() < 0.5
    window = rng.choice([0, 0, 0, 64])
    if op == "attend":
        return _tree(op, requests, heads, dtype, d, budget, nodes, group, page, ragged, window)
    return _tree(op, requests, heads, dtype, d, budget, nodes, group, page, ragged, window, scope=_log_int(rng, 1, budget),
                 path=min(nodes, rng.choice([1, 2, 4, 6, 8, 12])))


# ---------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _budgets(case):
    """The requests' budgets, and how many slots their units use: sizes of the case, not of the seed."""
    rng = random.Random("%(requests)d %(heads)d %(budget)d %(nodes)d" % case)
    most = case["budget"]
    budgets = [rng.randint(max(1, most // 4), most) if case["page"] and case["ragged"] else most for _ in range(case["requests"])]
    if case["requests"] > 1:
        budgets[0] = most
    used = [b if not case["ragged"] or rng.random() < 0.7 else rng.randint(b // 2, b) for b in budgets]
    return budgets, used


def _nodes(case):
    """Nodes of each request's tree."""
    rng = random.Random("%(requests)d %(nodes)d" % case)
    return [rng.randint((case["nodes"] + 1) // 2, case["nodes"]) if case["ragged"] else case["nodes"] for _ in range(case["requests"])]


def _trees(rng, case):
    """Parents of the nodes; -1: the last token of the cache."""
    T = case["nodes"]
    return [[-1 if i == 0 or rng.random() < 0.1 else rng.randint(max(0, i - 6), i - 1) for i in range(T)] for _ in range(case["requests"])]


def _paths(rng, case, parents, n_nodes):
    """The accepted nodes of every request, from the root on: most accept some, one in eight none."""
    paths = []
    for tree, n in zip(parents, n_nodes):
        i, path = rng.randint(n // 2, n - 1), []
        while i >= 0:
            path.insert(0, i)
            i = tree[i]
        paths.append([] if rng.random() < 0.125 else path[:case["path"]])
    return paths


def _prepare_tree(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    rng = random.Random(int(seed))
    R, H, G, T, B, d = (case[k] for k in ("requests", "heads", "group", "nodes", "budget", "head_dim"))
    U, dt = R * H, _dtype(case)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    u = randn(U, d)
    u /= u.norm(dim=1, keepdim=True)
    budgets, used = _budgets(case)
    n_nodes = _nodes(case)
    s = {"case": case}
    slots = B
    if case["page"]:
        # every request's pages lie anywhere in the pool, which has some more
        page = case["page"]
        M = -(-B // page)
        slots = M * page
        need = [-(-b // page) for b in budgets]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").cpu().tolist()
        table = [[order.pop() if j < k else -1 for j in range(M)] for k in need]
        s["table"], s["page"], s["n_pages"] = _ints(table), page, n_pages
        shape = (n_pages, H, page, d)
        heavy_u = u.view(R, H, d).mean(0)[None, :, None, :] * math.sqrt(R)  # (a page knows no request: a direction for each head)
        q_u = heavy_u.view(1, H, 1, d).expand(R, H, 1, d).reshape(U, 1, 1, d)
    else:
        shape = (U, B, d)
        heavy_u, q_u = u[:, None, :], u[:, None, None, :]
    K = randn(*shape)
    K += 4.0 * heavy_u * (rand(*shape[:-1], 1) < 0.02)
    s["K"], s["V"] = K.to(dt), randn(*shape).to(dt)
    del K
    s["q"] = (randn(U, T, G, d) + 2.0 * q_u).to(dt)
    s["k_new"], s["v_new"] = randn(U, T, d).to(dt), randn(U, T, d).to(dt)
    parents = _trees(rng, case)
    s["parent"], s["n_nodes"] = _ints(parents), _ints(n_nodes)
    s["budget"] = _ints(budgets)
    n_used = _ints(used).repeat_interleave(H)
    qpos0 = _ints([2 * B + rng.randint(0, 100) for _ in range(R)]).repeat_interleave(H)
    # the slots' positions: every second one or so, the newest just before the draft, in any order
    stored = torch.arange(B, device="cuda", dtype=torch.int32)
    pos = (qpos0[:, None] - 1 - 2 * stored - (rand(U, B) < 0.5).int()).gather(1, rand(U, B).argsort(1))
    pos = torch.where(stored < n_used[:, None], pos, -1)
    s["qpos0"], s["pos"], s["n_used"] = qpos0, pos, n_used
    s["scale"], s["bias"] = 1.0 / math.sqrt(d), 0.5 if case["window"] else 0.0
    if case["op"] == "commit":
        paths = _paths(rng, case, parents, n_nodes)
        A = case["path"]
        s["path"] = _ints([p + [0] * (A - len(p)) for p in paths])
        s["n_path"] = _ints([len(p) for p in paths])
        # tokens of very different ages and scores
        count = torch.randint(1, 3 * B + 2, (U, B), generator=g, device="cuda").float()
        mean = torch.exp(randn(U, B)) / B
        spread = mean * mean * torch.exp(2.0 * randn(U, B))
        stats = torch.stack([mean * count, (mean * mean + spread) * count, count], 1) * (stored < n_used[:, None])[:, None, :]
        # The state that a step changes, in one buffer: run() starts from the same one every time.
        ints = torch.cat([pos.reshape(-1), n_used])
        s["before"] = torch.cat([stats.reshape(-1), ints.view(torch.float32)])
        s["state"] = torch.empty_like(s["before"])
        k = stats.numel()
        s["stats"] = s["state"][:k].view(U, 3, B)
        s["pos"] = s["state"][k:k + U * B].view(torch.int32).view(U, B)
        s["n_used"] = s["state"][k + U * B:].view(torch.int32)
        s["state"].copy_(s["before"])
        s["lse"] = torch.empty((U, T, G), device="cuda")
        per = max(1, (1 << 27) // (T * G * max(slots, 1)))
        for at in range(0, U, per):  # the normalisers that the attention of the step has left
            s["lse"][at:at + per] = torch.logsumexp(_logits(s, at, min(U, at + per)), -1)
    if own:
        import paper_2402_06262_amd as roco
        s["params"] = roco.RocoParams(U, d, B, case.get("scope", 1), roco.ROCO_BF16 if case["dtype"] == "bf16" else roco.ROCO_F32, 0.0,
                                      case["window"], s["bias"])
        s["pages"] = roco.RocoPages(s["table"], s["n_pages"], s["page"], s["budget"]) if case["page"] else None
        s["workspace"] = torch.empty(max(16, roco.tree_workspace_bytes(s["params"], G, T)), dtype=torch.uint8, device="cuda")
        s["out"] = torch.zeros((U, T, G, d), dtype=dt, device="cuda")
        s["out_lse"] = torch.zeros((U, T, G), device="cuda")
        if case["op"] == "commit":
            s["evicted_slot"] = torch.empty((U, A), dtype=torch.int32, device="cuda")
            s["evicted_pos"] = torch.empty((U, A), dtype=torch.int32, device="cuda")
    return s


def _prepare_tables(case, seed):
    rng = random.Random("%(requests)d %(most)d %(grow)d" % case)  # lengths: sizes of the case
    R, page, most, grow = (case[k] for k in ("requests", "page", "most", "grow"))
    if grow:
        held = [rng.randint(0, most - 1) for _ in range(R)]
        want = [min(most, h + rng.randint(0, grow)) for h in held]
    else:
        held, want = [0] * R, [rng.randint(max(1, most // 4), most) for _ in range(R)]
    M = -(-most // page)
    taken = sum(-(-w // page) - -(-h // page) for h, w in zip(held, want))
    n_pages = taken + sum(-(-h // page) for h in held) + 8
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(M, device="cuda")
    n_held = -(-_ints(held) // page)
    start = torch.cumsum(n_held, 0) - n_held
    index = (start[:, None] + at).clamp(max=n_pages - 1)
    s = {"case": case, "held": _ints(held), "want": _ints(want),
         "table": torch.where(at < n_held[:, None], order[index], -1).to(torch.int32),
         "free": order[int(n_held.sum()):].contiguous()}
    s["page_start"] = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    s["row_start"] = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    new = [w - h for h, w in zip(held, want)]
    s["map"] = torch.zeros((R, max(1, max(new))) if case["padded"] else (max(1, sum(new)),), dtype=torch.int32, device="cuda")
    return s


def _prepare_store(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    rng = random.Random("%(groups)d %(rows)d" % case)
    N, rows, H, d, page = (case[k] for k in ("groups", "rows", "heads", "head_dim", "page"))
    dt = _dtype(case)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
    s = {"case": case}
    if N:
        fills = [rows] + [rng.randint(rows // 2, rows) for _ in range(N - 1)]
        s["K_rows"], s["V_rows"] = randn(N, H, rows, d), randn(N, H, rows, d)
        at = torch.arange(rows, device="cuda")
        need = -(-rows // page)
        n_pages = N * need + 2
        order = torch.randperm(n_pages, generator=g, device="cuda")[:N * need].view(N, need)
        slots = order[:, at // page] * page + at % page
        s["map"] = torch.where(at < _ints(fills)[:, None], slots, -1).to(torch.int32)
    else:
        # query, key and value heads of a token side by side; each token goes to a page of its own
        qkv = randn(rows, 3 * H, d)
        s["K_rows"], s["V_rows"] = qkv[:, H:2 * H], qkv[:, 2 * H:]
        n_pages = rows + 2
        order = torch.randperm(n_pages, generator=g, device="cuda")[:rows]
        s["map"] = (order * page + torch.randint(0, page, (rows,), generator=g, device="cuda")).to(torch.int32)
    s["K_pool"], s["V_pool"] = (torch.zeros((n_pages, H, page, d), dtype=dt, device="cuda") for _ in range(2))
    return s


def prepare(case, seed):
    if case["op"] == "tables":
        return _prepare_tables(case, seed)
    if case["op"] == "store":
        return _prepare_store(case, seed)
    return _prepare_tree(case, seed)


# ---------------------------------------------------------------------------------------------- plain forms
def _rows(s, cache, a, b):
    """Rows of units a .. b - 1 in 32 bits, [b - a, slots, d]."""
    if "table" not in s:
        return cache[a:b].float()
    H, B = s["case"]["heads"], s["case"]["budget"]
    u = torch.arange(a, b, device="cuda")
    rows = cache[s["table"][u // H].clamp(min=0).long(), (u % H)[:, None]]  # [units, pages, page, d]
    return rows.flatten(1, 2)[:, :B].float()


def _ancestors(s):
    """[requests, T, T]: node i sees node j, itself or one above it."""
    T = s["parent"].shape[1]
    i = torch.arange(T, device="cuda")
    sees = (i[:, None] == i).expand(len(s["parent"]), T, T)
    up = s["parent"].long()
    for _ in range(T.bit_length()):  # twice as far up each time, all nodes of all trees at once; -1: above the roots
        there = up.clamp(min=0)
        sees = sees | (sees.gather(1, there[:, :, None].expand_as(sees)) & (up >= 0)[:, :, None])
        up = torch.where(up >= 0, up.gather(1, there), -1)
    return sees


def _logits(s, a, b):
    """Scaled logits of units a .. b - 1, [units, T, group, slots + T]; what a row does not see is -inf."""
    case = s["case"]
    H, T, G, d = case["heads"], case["nodes"], case["group"], case["head_dim"]
    r = torch.arange(a, b, device="cuda") // H
    q = s["q"][a:b].float().flatten(1, 2) * s["scale"]
    K = torch.cat([_rows(s, s["K"], a, b), s["k_new"][a:b].float()], 1)
    x = torch.bmm(q, K.transpose(1, 2).contiguous()).view(b - a, T, G, -1)
    B = x.shape[-1] - T
    sees = _ancestors(s)
    if case["window"]:
        depth = sees.sum(-1)[r] - 1
        away = (s["qpos0"][a:b, None] + depth)[:, :, None] - torch.cat([s["pos"][a:b], s["qpos0"][a:b, None] + depth], 1)[:, None, :]
        x = x + s["bias"] * ((away >= 0) & (away < case["window"]))[:, :, None, :]
    slots = (torch.arange(B, device="cuda") < s["n_used"][a:b, None])[:, None, :].expand(-1, T, -1)
    nodes = sees[r] & (torch.arange(T, device="cuda") < s["n_nodes"][r, None])[:, None, :]
    return x.masked_fill(~torch.cat([slots, nodes], 2)[:, :, None, :], -math.inf)


def _plain_attend(s):
    case = s["case"]
    U, T, G, d = s["q"].shape
    x = _logits(s, 0, U)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    V = torch.cat([_rows(s, s["V"], 0, U), s["v_new"].float()], 1)
    out = (torch.bmm(p.flatten(1, 2), V).view(U, T, G, d) / total).to(s["q"].dtype)
    lse = (m + torch.log(total)).squeeze(-1)
    # rows behind a tree's last node are not written: zeros, as they were
    there = (torch.arange(T, device="cuda") < s["n_nodes"].repeat_interleave(case["heads"])[:, None])[:, :, None]
    return out * there[..., None], torch.where(there, lse, 0.0)


def _rank(keys):
    """Place of every element among its row's, the lowest first, equal ones in order."""
    order = keys.argsort(dim=1, stable=True)
    return torch.empty_like(order).scatter_(1, order, torch.arange(keys.shape[1], device="cuda").expand_as(order))


def _plain_commit(s):
    case = s["case"]
    H, B, A, d = case["heads"], case["budget"], case["path"], case["head_dim"]
    s["state"].copy_(s["before"])
    stats, pos, n_used = s["stats"], s["pos"], s["n_used"]
    U = len(n_used)
    r = torch.arange(U, device="cuda") // H
    unit = torch.arange(U, device="cuda")[:, None]
    n, a = n_used.long(), s["n_path"][r].long()
    most = s["budget"][r].long()
    slot, k = torch.arange(B, device="cuda"), torch.arange(A, device="cuda")
    n_new = torch.minimum(most, n + a)
    evict = (n + a - n_new)[:, None]
    # victims by the statistics as they stand, each operation rounded on its own
    held = slot < n[:, None]
    score = (stats[:, 0].double() / stats[:, 2].double()).float()
    spread = (stats[:, 1].double() / stats[:, 2].double()).float() - score * score
    spread = torch.where(held, spread.clamp(min=0.0), math.inf)
    scope = torch.minimum(torch.minimum(torch.full_like(most, case["scope"]), most) + evict[:, 0] - 1, n)[:, None]
    inside = (_rank(spread) < scope) & held
    victim = _rank(torch.where(inside, score, math.inf)) < evict
    taken = victim | (~held & (slot < n_new[:, None]))
    # the accepted tokens go to the taken slots in order
    order = (~taken).long().argsort(dim=1, stable=True)[:, :A]
    if order.shape[1] < A:
        order = torch.nn.functional.pad(order, (0, A - order.shape[1]))
    real = k < a[:, None]
    was = held.gather(1, order) & real
    evicted_slot = torch.where(was, order, -1).to(torch.int32)
    evicted_pos = torch.where(was, pos.gather(1, order), -1).to(torch.int32)
    # probabilities of the accepted rows, the mean of their heads
    node = s["path"][r].long()
    x = _logits_of_path(s, r, unit, node, n)
    p = torch.exp(x - s["lse"][unit, node][..., None]).mean(2) * real[:, :, None]  # [units, A, B + A]
    keep = (held & ~taken)[:, None, :]
    old = p[:, :, :B]
    sums = torch.stack([old.sum(1), (old * old).sum(1), a[:, None].expand(-1, B).float()], 1)
    new = p[:, :, B:]
    fresh = torch.stack([new.sum(1), (new * new).sum(1), (a[:, None] - k).float()], 1)
    stats.copy_(torch.where(keep, stats + sums, torch.where(taken[:, None, :], 0.0, stats)))
    at_unit, at_k = real.nonzero(as_tuple=True)
    at_slot = order[at_unit, at_k]
    stats[at_unit, :, at_slot] = fresh[at_unit, :, at_k]
    pos[at_unit, at_slot] = s["qpos0"][at_unit] + at_k.to(torch.int32)
    n_used.copy_(n_new)
    at_node = node[at_unit, at_k]
    for cache, rows in ((s["K"], s["k_new"]), (s["V"], s["v_new"])):
        if "table" in s:
            cache[s["table"][r[at_unit], at_slot // s["page"]].long(), at_unit % H, at_slot % s["page"]] = rows[at_unit, at_node]
        else:
            cache[at_unit, at_slot] = rows[at_unit, at_node]
    return _committed(s, evicted_slot, evicted_pos)


def _committed(s, evicted_slot, evicted_pos):
    """What a commit leaves; the planes of the statistics are values of different kinds."""
    acc, acc2, count = s["stats"].unbind(1)
    return {"K": s["K"], "V": s["V"], "acc": acc, "acc2": acc2, "count": count, "pos": s["pos"], "n_used": s["n_used"],
            "evicted_slot": evicted_slot, "evicted_pos": evicted_pos}


def _logits_of_path(s, r, unit, node, n):
    """Scaled logits of the accepted rows over the old slots and the accepted tokens, [units, A, group, B + A]."""
    case = s["case"]
    U, A = node.shape
    G, B, d = case["group"], case["budget"], case["head_dim"]
    q = s["q"][unit, node].float().flatten(1, 2) * s["scale"]
    K = torch.cat([_rows(s, s["K"], 0, U), s["k_new"][unit, node].float()], 1)
    x = torch.bmm(q, K.transpose(1, 2).contiguous()).view(U, A, G, B + A)
    k = torch.arange(A, device="cuda")
    if case["window"]:
        mine = s["qpos0"][:, None] + k
        away = mine[:, :, None] - torch.cat([s["pos"], mine], 1)[:, None, :]
        x = x + s["bias"] * ((away >= 0) & (away < case["window"]))[:, :, None, :]
    slots = (torch.arange(B, device="cuda") < n[:, None])[:, None, :].expand(-1, A, -1)
    causal = (k[:, None] >= k).expand(U, A, A)
    return x.masked_fill(~torch.cat([slots, causal], 2)[:, :, None, :], -math.inf)


def _plain_tables(s):
    case = s["case"]
    page, table, free = case["page"], s["table"], s["free"]
    R, M = table.shape
    held, want = s["held"].long(), s["want"].long()
    first, last = -(-held // page), -(-want // page)
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    page_start = torch.cat([zero, torch.cumsum(last - first, 0)])
    row_start = torch.cat([zero, torch.cumsum(want - held, 0)])
    j = torch.arange(M, device="cuda")
    index = page_start[:R, None] + j - first[:, None]
    taken = torch.where(index < len(free), free[index.clamp(0, len(free) - 1)], -1)
    table = torch.where((j >= first[:, None]) & (j < last[:, None]), taken, table)
    rows = s["map"].shape[-1]
    i = torch.arange(rows, device="cuda")
    if case["padded"]:
        request = torch.arange(R, device="cuda")[:, None].expand(R, rows)
        slot = held[:, None] + i
        real = slot < want[:, None]
    else:
        request = (torch.searchsorted(row_start, i, right=True) - 1).clamp(0, R - 1)
        slot = held[request] + i - row_start[request]
        real = i < row_start[R]
    at = table[request, (slot // page).clamp(0, M - 1)]
    slots = torch.where(real & (at >= 0), at * page + slot % page, -1)
    return {"table": table.to(torch.int32), "page_start": page_start.to(torch.int32), "row_start": row_start.to(torch.int32),
            "map": slots.to(torch.int32)}


def _plain_store(s):
    page, slots = s["case"]["page"], s["map"].long()
    for pool, rows in ((s["K_pool"], s["K_rows"]), (s["V_pool"], s["V_rows"])):
        rows = rows.permute(0, 2, 1, 3) if s["case"]["groups"] else rows
        real = slots >= 0
        at = slots[real]
        pool[at // page, :, at % page] = rows[real]
    return s["K_pool"], s["V_pool"]


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if not own:
        return {"attend": _plain_attend, "commit": _plain_commit, "tables": _plain_tables, "store": _plain_store}[case["op"]](s)
    import paper_2402_06262_amd as roco
    if case["op"] == "attend":
        roco.roco_tree_attend(s["params"], case["heads"], case["group"], case["nodes"], s["pages"], s["q"], s["k_new"], s["v_new"], s["parent"],
                              s["n_nodes"], s["qpos0"], s["K"], s["V"], s["pos"], s["n_used"], s["out"], s["out_lse"], s["workspace"])
        return s["out"], s["out_lse"]
    if case["op"] == "commit":
        s["state"].copy_(s["before"])
        roco.roco_tree_commit(s["params"], case["heads"], case["group"], case["nodes"], s["pages"], s["q"], s["k_new"], s["v_new"], s["lse"],
                              case["path"], s["path"], s["n_path"], s["qpos0"], s["K"], s["V"], s["stats"], s["pos"], s["n_used"],
                              s["evicted_slot"], s["evicted_pos"], s["workspace"])
        return _committed(s, s["evicted_slot"], s["evicted_pos"])
    if case["op"] == "tables":
        roco.roco_page_tables(s["held"], s["want"], case["page"], s["free"], s["table"], s["page_start"], s["row_start"], s["map"])
        return {k: s[k] for k in ("table", "page_start", "row_start", "map")}
    roco.roco_page_store(s["K_rows"], s["V_rows"], s["map"], s["K_pool"], s["V_pool"])
    return s["K_pool"], s["V_pool"]


def work(case):
    if case["op"] == "tables":
        rng = random.Random("%(requests)d %(most)d %(grow)d" % case)
        R, page, most, grow = (case[k] for k in ("requests", "page", "most", "grow"))
        if grow:
            held = [rng.randint(0, most - 1) for _ in range(R)]
            want = [min(most, h + rng.randint(0, grow)) for h in held]
        else:
            held, want = [0] * R, [rng.randint(max(1, most // 4), most) for _ in range(R)]
        new = [w - h for h, w in zip(held, want)]
        taken = sum(-(-w // page) - -(-h // page) for h, w in zip(held, want))
        return {"bytes": 4.0 * (2 * R + 2 * taken + 2 * (R + 1) + (R * max(1, max(new)) if case["padded"] else max(1, sum(new)))), "flops": 0}
    e = 2 if case["dtype"] == "bf16" else 4
    H, d = case["heads"], case["head_dim"]
    if case["op"] == "store":
        rng = random.Random("%(groups)d %(rows)d" % case)
        N, rows = case["groups"], case["rows"]
        total = rows + sum(rng.randint(rows // 2, rows) for _ in range(N - 1)) if N else rows
        return {"bytes": 4.0 * total * H * d * e + 4.0 * max(1, N) * rows, "flops": 0}
    _, used = _budgets(case)
    nodes = _nodes(case)
    G, T = case["group"], case["nodes"]
    slots = float(H * sum(used))
    if case["op"] == "attend":
        rows = H * G * sum(nodes)
        seen = float(H * G * sum(t * (n + min(t, 6)) for t, n in zip(nodes, used)))
        return {"bytes": slots * 2 * d * e + 2 * rows * d * e + 4 * rows + 2 * H * sum(nodes) * d * e + (4 * slots if case["window"] else 0),
                "flops": 4 * seen * d}
    a = min(case["path"], 4)  # accepted tokens of a request, or so
    return {"bytes": slots * (d * e + 24) + H * case["requests"] * a * (4 + G) * d * e, "flops": 2 * slots * a * G * d}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _exact_rows(s, cache, u, n):
    """The first n rows of unit u."""
    if "table" not in s:
        return cache[u, :n].double()
    H, page = s["case"]["heads"], s["page"]
    pages = s["table"][u // H, :-(-n // page)].tolist()
    return torch.cat([cache[p, u % H] for p in pages] + [cache[0, 0, :0]])[:n].double()


def _exact_seen(parents, n):
    """For every node the list of the nodes it sees."""
    seen = []
    for i in range(n):
        seen.append((seen[parents[i]] if parents[i] >= 0 else []) + [i])
    return seen


def _exact_attend(s):
    case = s["case"]
    U, T, G, d = s["q"].shape
    H, w = case["heads"], case["window"]
    out = torch.zeros((U, T, G, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((U, T, G), dtype=torch.float64, device="cuda")
    parents, nodes, used = s["parent"].tolist(), s["n_nodes"].tolist(), s["n_used"].tolist()
    start = s["qpos0"].tolist()
    for u in range(U):
        r, n = u // H, used[u]
        t = nodes[r]
        if u % H == 0:
            seen = _exact_seen(parents[r], t)
            mask = torch.zeros((t, t), dtype=torch.bool)
            for i, js in enumerate(seen):
                mask[i, js] = True
            mask = mask.cuda()
            depth = torch.tensor([len(js) - 1 for js in seen], device="cuda")
        keys = torch.cat([_exact_rows(s, s["K"], u, n), s["k_new"][u, :t].double()])
        values = torch.cat([_exact_rows(s, s["V"], u, n), s["v_new"][u, :t].double()])
        x = (s["q"][u, :t].double().reshape(t * G, d) @ keys.t()).view(t, G, n + t) / math.sqrt(d)
        if w:
            at = torch.cat([s["pos"][u, :n].long(), start[u] + depth])
            gap = (start[u] + depth)[:, None] - at
            x += s["bias"] * ((gap >= 0) & (gap < w))[:, None, :]
        x[:, :, n:].masked_fill_(~mask[:, None, :], -math.inf)
        z = torch.logsumexp(x, -1)
        out[u, :t] = (torch.exp(x - z[..., None]).view(t * G, n + t) @ values).view(t, G, d)
        lse[u, :t] = z
    return out, lse


def _exact_commit(s):
    case = s["case"]
    H, B, G, d, w = case["heads"], case["budget"], case["group"], case["head_dim"], case["window"]
    stats = s["stats"].cpu().numpy()
    result = stats.astype(np.float64)
    pos, used, budgets = s["pos"].cpu().numpy(), s["n_used"].tolist(), s["budget"].tolist()
    paths, lengths, start = s["path"].tolist(), s["n_path"].tolist(), s["qpos0"].tolist()
    for u in range(len(used)):
        r, n = u // H, used[u]
        a, most = lengths[r], budgets[r]
        if a == 0:
            continue
        n_new = min(most, n + a)
        E = n + a - n_new
        victims = np.zeros(0, dtype=np.int64)
        if E:
            acc, acc2, cnt = stats[u, :, :n]  # (the choice is defined on 32-bit keys)
            score = acc / cnt
            spread = np.maximum(acc2 / cnt - score * score, np.float32(0))
            scope = np.sort(np.argsort(spread, kind="stable")[:min(n, min(case["scope"], most) + E - 1)])
            victims = scope[np.argsort(score[scope], kind="stable")[:E]]
        slots = sorted(victims.tolist()) + list(range(n, n_new))
        node = paths[r][:a]
        keys = torch.cat([_exact_rows(s, s["K"], u, n), s["k_new"][u, node].double()])
        x = (s["q"][u, node].double().reshape(a * G, d) @ keys.t()).view(a, G, n + a) / math.sqrt(d)
        mine = start[u] + torch.arange(a, device="cuda")
        if w:
            gap = mine[:, None] - torch.cat([torch.from_numpy(pos[u, :n]).cuda().long(), mine])
            x += s["bias"] * ((gap >= 0) & (gap < w))[:, None, :]
        x[:, :, n:].masked_fill_(torch.ones((a, a), dtype=torch.bool, device="cuda").triu(1)[:, None, :], -math.inf)
        p = torch.exp(x - s["lse"][u, node].double()[..., None]).mean(1)
        sums = torch.stack([p.sum(0), (p * p).sum(0)]).cpu().numpy()
        result[u, :2, :n] += sums[:, :n]
        result[u, 2, :n] += a
        for k, j in enumerate(slots):
            result[u, :2, j] = sums[:, n + k]
            result[u, 2, j] = a - k
    acc, acc2, count = torch.from_numpy(result).unbind(1)
    return {"K": None, "V": None, "acc": acc, "acc2": acc2, "count": count, "pos": None, "n_used": None, "evicted_slot": None,
            "evicted_pos": None}


def _exact_store(s):
    pools = []
    for rows in (s["K_rows"], s["V_rows"]):
        pool = torch.zeros(s["K_pool"].shape, dtype=torch.float64, device="cuda")
        N, H, page, d = pool.shape
        rows = rows.double()
        tokens = rows.transpose(1, 2).reshape(-1, H, d) if rows.dim() == 4 else rows
        where = s["map"].reshape(-1).long()
        kept = torch.nonzero(where >= 0).squeeze(1)
        flat = ((where[kept] // page)[:, None] * H + torch.arange(H, device="cuda")) * page + (where[kept] % page)[:, None]
        pool.view(-1, d).index_copy_(0, flat.reshape(-1), tokens[kept].reshape(-1, d))
        pools.append(pool)
    return tuple(pools)


def exact(case, seed):
    if case["op"] == "tables":
        return None
    s = prepare(case, seed)
    if case["op"] == "store":
        return _exact_store(s)
    return _exact_attend(s) if case["op"] == "attend" else _exact_commit(s)
