"""Chunks of new tokens over budgeted caches, and the verification of drafted tokens: what is measured of the operators roco_chunk_attend,
roco_chunk_commit and roco_tree_verify, beside their plain forms.

A case is a plain dict; `op` names the operator.  Caches and queries follow the heavy-hitter recipe of `inputs/`: N(0, 1) rows, a unit vector u
per head, 4 u added to 2 % of the keys and 2 u to every query; the chunks' rows lie as a fused projection leaves them, query, key and value
heads of a token side by side.  Probabilities are softmaxes of N(0, 4^2) logits, the target's without its smallest values, as a sampler's
filter leaves them; the draft's logits are the target's with N(0, 1) added, and drafted tokens are drawn from the draft's probabilities.
`own` false: elementary torch operations in 32 bits (probabilities' sums in 64); `own` true: the library's calls.
"""
import math
import random

import torch

own = False


# ---------------------------------------------------------------------------------------------- cases
def _chunk(op, requests, heads, group, dtype, head_dim, budget, chunk, page=0, ragged=False, single=0.0, window=0, scope=64, name=None):
    """Chunks of up to `chunk` tokens of `requests` requests, a share `single` of which decode a token each; page > 0: caches in pages, with
    a budget of each request's own; ragged: caches and chunks of different lengths."""
    c = {"op": op, "requests": requests, "heads": heads, "group": group, "dtype": dtype, "head_dim": head_dim, "budget": budget, "chunk": chunk,
         "page": page, "ragged": ragged, "single": single, "window": window}
    if op == "commit":
        c["scope"] = scope
    if name is not None:
        c["name"] = name
    return c


def _verify(requests, nodes, vocab, children=1, drafts="sampled", dtype="f32", ragged=False, name=None):
    """Trees of up to `children` continuations of a node (1: chains).  drafts: "sampled" (each drawn on its own), "distinct" (the
    continuations of a node differ) or "given" (without probabilities: copied from a prompt, say)."""
    c = {"op": "verify", "requests": requests, "nodes": nodes, "vocab": vocab, "children": children, "drafts": drafts, "dtype": dtype,
         "ragged": ragged}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a token of each of four requests of a tiny fp32 layer: nothing but latency
        _chunk("attend", 4, 4, 1, "f32", 64, 500, 1, name="attend_one_token"),
        # the next 512 tokens of four prompts of a grouped model, over caches that are full already
        _chunk("attend", 4, 8, 4, "bf16", 128, 4096, 512, page=64, name="attend_prompts"),
        # a server's step: most requests decode, the others feed their prompts; paged caches of different budgets
        _chunk("attend", 24, 8, 4, "bf16", 128, 4096, 384, page=16, ragged=True, single=0.75, name="attend_mixed"),
        # a part of a long document over a long cache
        _chunk("attend", 1, 8, 4, "bf16", 128, 32768, 1024, page=256, name="attend_long"),
        # head_dim 64, dense caches, one query head per key/value head, a recency window
        _chunk("attend", 6, 12, 1, "bf16", 64, 2048, 333, ragged=True, window=64, name="attend_window"),
        # full precision, odd sizes
        _chunk("attend", 5, 5, 3, "f32", 128, 1501, 101, ragged=True, name="attend_ragged_f32"),
        # 16 tokens of a tiny fp32 layer taken over: latency
        _chunk("commit", 4, 4, 1, "f32", 64, 500, 16, scope=32, name="commit_tiny_f32"),
        # the same 512 tokens of four prompts taken over
        _chunk("commit", 4, 8, 4, "bf16", 128, 4096, 512, page=64, name="commit_prompts"),
        # caches and chunks of different lengths, head_dim 64, eight query heads per key/value head
        _chunk("commit", 12, 8, 8, "bf16", 64, 2048, 200, page=32, ragged=True, scope=512, name="commit_ragged"),
        # one request's five drafted tokens: latency
        _verify(1, 6, 32000, name="verify_one"),
        # drafted chains of a full batch, an odd vocabulary
        _verify(64, 8, 100003, ragged=True, name="verify_chains"),
        # trees of 32 nodes whose siblings differ
        _verify(32, 32, 65536, children=3, drafts="distinct", name="verify_trees"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "commit", "verify"])
    if op == "verify":
        nodes, vocab = _log_int(rng, 1, 64), _log_int(rng, 1000, 131072)
        dtype = rng.choice(["f32", "f32", "bf16"])
        requests = _log_int(rng, 1, max(1, min(128, (1 << 26) // (nodes * vocab))))
        return _verify(requests, nodes, vocab, rng.choice([1, 1, 2, 3, 5]), rng.choice(["sampled", "distinct", "given"]), dtype, rng.random() < 0.5)
    dtype, d = rng.choice([("bf16", 128), ("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
    e = 2 if dtype == "bf16" else 4
    heads, group = rng.choice([1, 2, 5, 8, 8, 16]), rng.choice([1, 1, 2, 3, 4, 8])
    budget = _log_int(rng, 64, 16384)
    chunk = _log_int(rng, 1, 2048)
    if op == "commit":
        chunk = min(chunk, budget)
    # at most the products of the longest listed cache (fp32: a sixteenth of them), and a cache's bytes
    rows = heads * group * chunk
    most = min((1 << 30) // (rows * (budget + chunk) * d // 128 * (1 if e == 2 else 16) + 1), (512 << 20) // (2 * budget * heads * d * e))
    if most < 1:
        chunk = max(1, (1 << 30) // (heads * group * (budget + chunk) * d // 128 * (1 if e == 2 else 16)))
    requests = _log_int(rng, 1, max(1, min(32, most)))
    return _chunk(op, requests, heads, group, dtype, d, budget, chunk, rng.choice([0, 0, 16, 64, 128]), rng.random() < 0.6, rng.choice([0.0, 0.0, 0.75]),
                  rng.choice([0, 0, 0, 64]), scope=_log_int(rng, 1, budget))


# ---------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _lengths(case):
    """The requests' budgets, the slots that their units use and their chunks' tokens: sizes of the case, not of the seed."""
    rng = random.Random("%(requests)d %(heads)d %(budget)d %(chunk)d" % case)
    most, chunk = case["budget"], case["chunk"]
    budgets = [rng.randint(max(1, most // 4), most) if case["page"] and case["ragged"] else most for _ in range(case["requests"])]
    budgets[0] = most
    used = [b if not case["ragged"] or rng.random() < 0.5 else rng.randint(0, b) for b in budgets]
    tokens = [1 if rng.random() < case["single"] else rng.randint(0, chunk) if case["ragged"] and not case["single"] else chunk for _ in budgets]
    tokens[0] = chunk
    if case["op"] == "commit":
        tokens = [min(t, b) for t, b in zip(tokens, budgets)]
    return budgets, used, tokens


def _prepare_chunk(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    rng = random.Random(int(seed))
    R, H, G, B, d = (case[k] for k in ("requests", "heads", "group", "budget", "head_dim"))
    U, dt = R * H, _dtype(case)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    u = randn(H, d)
    u /= u.norm(dim=1, keepdim=True)
    budgets, used, tokens = _lengths(case)
    total = sum(tokens)
    s = {"case": case}
    if case["page"]:
        # every request's pages lie anywhere in the pool, which has some more
        page = case["page"]
        M = -(-B // page)
        need = [-(-b // page) for b in budgets]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").cpu().tolist()
        table = [[order.pop() if j < k else -1 for j in range(M)] for k in need]
        s["table"], s["page"], s["n_pages"] = _ints(table), page, n_pages
        shape, heavy = (n_pages, H, page, d), u[:, None, :]
    else:
        shape, heavy = (U, B, d), u.repeat(R, 1)[:, None, :]
    K = randn(*shape)
    K += 4.0 * heavy * (rand(*shape[:-1], 1) < 0.02)
    s["K"], s["V"] = K.to(dt), randn(*shape).to(dt)
    del K
    # query, key and value heads of a token side by side
    qkv = randn(total, H * G + 2 * H, d)
    qkv[:, :H * G] += 2.0 * u.repeat_interleave(G, 0)
    qkv = qkv.to(dt)
    s["q"], s["k_new"], s["v_new"] = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
    start = [0]
    for t in tokens:
        start.append(start[-1] + t)
    s["start"], s["budget"] = _ints(start), _ints(budgets)
    s["n_used"] = _ints(used).repeat_interleave(H)
    s["qpos0"] = _ints([2 * B + rng.randint(0, 100) for _ in range(R)])
    # the slots' positions: every second one or so, the newest just before the chunk, in any order
    stored = torch.arange(B, device="cuda", dtype=torch.int32)
    first = s["qpos0"].repeat_interleave(H)[:, None]
    pos = (first - 1 - 2 * stored - (rand(U, B) < 0.5).int()).gather(1, rand(U, B).argsort(1))
    s["pos"] = torch.where(stored < s["n_used"][:, None], pos, -1)
    s["scale"], s["bias"] = 1.0 / math.sqrt(d), 0.5 if case["window"] else 0.0
    s["longest"] = max(tokens)
    if case["op"] == "commit":
        # tokens of very different ages and scores
        count = torch.randint(1, 3 * B + 2, (U, B), generator=g, device="cuda").float()
        mean = torch.exp(randn(U, B)) / B
        spread = mean * mean * torch.exp(2.0 * randn(U, B))
        stats = torch.stack([mean * count, (mean * mean + spread) * count, count], 1) * (stored < s["n_used"][:, None])[:, None, :]
        # The state that a step changes, in one buffer: run() starts from the same one every time.
        ints = torch.cat([s["pos"].reshape(-1), s["n_used"]])
        s["before"] = torch.cat([stats.reshape(-1), ints.view(torch.float32)])
        s["state"] = s["before"].clone()
        k = stats.numel()
        s["stats"] = s["state"][:k].view(U, 3, B)
        s["pos"] = s["state"][k:k + U * B].view(torch.int32).view(U, B)
        s["n_used"] = s["state"][k + U * B:].view(torch.int32)
        # the normalisers that the attention of the step has left
        s["lse"] = torch.zeros((total, H * G), device="cuda")
        for r in range(R):
            x = _logits(s, r, r + 1)
            s["lse"][start[r]:start[r + 1]] = torch.logsumexp(x, -1).permute(0, 2, 1, 3).reshape(-1, H * G)[:tokens[r]]
    if own:
        import paper_2402_06262_amd as roco
        s["params"] = roco.RocoParams(U, d, B, case.get("scope", 1), roco.ROCO_BF16 if case["dtype"] == "bf16" else roco.ROCO_F32, 0.0,
                                      case["window"], s["bias"])
        s["pages"] = roco.RocoPages(s["table"], s["n_pages"], s["page"], s["budget"]) if case["page"] else None
        s["workspace"] = torch.empty(max(16, roco.chunk_workspace_bytes(s["params"], H, G, total)), dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty((total, H * G, d), dtype=dt, device="cuda")
        s["out_lse"] = torch.empty((total, H * G), device="cuda")
        if case["op"] == "commit":
            s["evicted_slot"] = torch.empty((total, H), dtype=torch.int32, device="cuda")
            s["evicted_pos"] = torch.empty((total, H), dtype=torch.int32, device="cuda")
    return s


def _parents(case, rng):
    T, kids = case["nodes"], case["children"]
    return [[-1] + [max(0, (i - 1) // kids - (rng.randint(0, 1) if kids > 1 else 0)) for i in range(1, T)] for _ in range(case["requests"])]


def _prepare_verify(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    rng = random.Random(int(seed))
    R, T, V, dt = case["requests"], case["nodes"], case["vocab"], _dtype(case)
    p = torch.empty((R, T, V), dtype=dt, device="cuda")
    q = torch.empty((R, T, V), dtype=dt, device="cuda")
    parents = _parents(case, rng)
    parent = torch.tensor(parents, device="cuda")
    # which of its parent's continuations a node is
    place = torch.tensor([[sum(row[j] == row[i] for j in range(i)) for i in range(T)] for row in parents], device="cuda")
    kids = min(V, int(place.max()) + 1)
    tokens = torch.zeros((R, T), dtype=torch.int32, device="cuda")
    for r in range(R):
        logits = 4.0 * torch.randn((T, V), generator=g, device="cuda")
        target = torch.softmax(logits, -1)
        target = target * (target > 1e-3 * target.amax(-1, keepdim=True))
        p[r] = (target / target.sum(-1, keepdim=True)).to(dt)
        draft = torch.softmax(logits + torch.randn((T, V), generator=g, device="cuda"), -1)
        q[r] = draft.to(dt)
        if case["drafts"] == "sampled":
            drawn = torch.multinomial(draft, kids, replacement=True, generator=g)
        else:  # the first to arrive of races with these rates
            drawn = (draft / torch.empty_like(draft).exponential_(generator=g)).topk(kids, -1).indices
        tokens[r] = drawn[parent[r].clamp(min=0), place[r].clamp(max=kids - 1)].int()
    s = {"case": case, "p": p, "q": None if case["drafts"] == "given" else q, "tokens": tokens,
         "parent": None if case["children"] == 1 else parent.int()}
    sizes = random.Random("%(requests)d %(nodes)d" % case)
    s["n_nodes"] = _ints([sizes.randint((T + 1) // 2, T) if case["ragged"] else T for _ in range(R)])
    s["accept"] = torch.rand((R, T), generator=g, device="cuda")
    s["choose"] = torch.rand((R,), generator=g, device="cuda")
    s["path"], s["n_path"], s["next"] = _ints([[0] * T] * R), _ints([0] * R), _ints([0] * R)
    if own:
        import paper_2402_06262_amd as roco
        s["workspace"] = torch.empty(max(16, roco.verify_workspace_bytes(R, T, V)), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return _prepare_verify(case, seed) if case["op"] == "verify" else _prepare_chunk(case, seed)


# ---------------------------------------------------------------------------------------------- plain forms
def _cache_rows(s, cache, a, b):
    """Rows of the units of requests a .. b - 1 in 32 bits, [b - a, heads, budget, d]."""
    H, B = s["case"]["heads"], s["case"]["budget"]
    if "table" not in s:
        return cache.view(-1, H, B, cache.shape[-1])[a:b].float()
    rows = cache[s["table"][a:b].clamp(min=0).long()]  # [requests, pages, heads, page, d]
    return rows.transpose(1, 2).flatten(2, 3)[:, :, :B].float()


def _places(s, a, b):
    """Where the tokens of requests a .. b - 1 lie in the packed rows, padded, and which of them there are: [b - a, longest]."""
    i = torch.arange(s["longest"], device="cuda")
    at = s["start"][a:b, None] + i
    return at.clamp(max=len(s["q"]) - 1).long(), at < s["start"][a + 1:b + 1, None]


def _logits(s, a, b):
    """Scaled logits of requests a .. b - 1, [b - a, heads, longest, group, budget + longest]; what a row does not see is -inf."""
    case = s["case"]
    H, G, B, d, C = case["heads"], case["group"], case["budget"], case["head_dim"], s["longest"]
    at, real = _places(s, a, b)
    q = s["q"][at].float().view(b - a, C, H, G, d).permute(0, 2, 1, 3, 4).reshape(-1, C * G, d) * s["scale"]
    K = torch.cat([_cache_rows(s, s["K"], a, b), s["k_new"][at].float().transpose(1, 2)], 2).flatten(0, 1)
    x = torch.bmm(q, K.transpose(1, 2).contiguous()).view(b - a, H, C, G, B + C)
    i = torch.arange(C, device="cuda")
    if case["window"]:
        mine = (s["qpos0"][a:b, None] + i)[:, None, :].expand(-1, H, -1)
        away = mine[..., None] - torch.cat([s["pos"].view(-1, H, B)[a:b], mine], 2)[:, :, None, :]
        x = x + s["bias"] * ((away >= 0) & (away < case["window"]))[:, :, :, None, :]
    slots = torch.arange(B, device="cuda") < s["n_used"].view(-1, H)[a:b, :, None]
    seen = torch.cat([slots[:, :, None, :].expand(-1, -1, C, -1), ((i <= i[:, None]) & real[:, None, :])[:, None].expand(-1, H, -1, -1)], 3)
    return x.masked_fill_(~seen[:, :, :, None, :], -math.inf)


def _plain_attend(s):
    case = s["case"]
    R, H, G, d, C = case["requests"], case["heads"], case["group"], case["head_dim"], s["longest"]
    at, real = _places(s, 0, R)
    x = _logits(s, 0, R)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)  # (a row of padding may see nothing)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    V = torch.cat([_cache_rows(s, s["V"], 0, R), s["v_new"][at].float().transpose(1, 2)], 2).flatten(0, 1)
    out = torch.bmm(p.flatten(0, 1).flatten(1, 2), V).view(R, H, C, G, d) / total
    lse = m + torch.log(total)
    back = lambda t: t.permute(0, 2, 1, 3, 4).reshape(R, C, H * G, -1)[real]  # noqa: E731
    return back(out).to(s["q"].dtype), back(lse).squeeze(-1)


def _rank(keys):
    """Place of every element among its row's, the lowest first, equal ones in order."""
    order = keys.argsort(dim=1, stable=True)
    return torch.empty_like(order).scatter_(1, order, torch.arange(keys.shape[1], device="cuda").expand_as(order))


def _plain_commit(s):
    case = s["case"]
    R, H, B, C = case["requests"], case["heads"], case["budget"], s["longest"]
    s["state"].copy_(s["before"])
    stats, pos, n_used = s["stats"], s["pos"], s["n_used"]
    U = R * H
    r = torch.arange(U, device="cuda") // H
    at, real = _places(s, 0, R)
    n, c = n_used.long(), (s["start"][1:] - s["start"][:-1]).long()[r]
    most = s["budget"][r].long()
    slot, k = torch.arange(B, device="cuda"), torch.arange(C, device="cuda")
    n_new = torch.minimum(most, n + c)
    evict = (n + c - n_new)[:, None]
    # victims by the statistics as they stand, each operation rounded on its own
    held = slot < n[:, None]
    score = (stats[:, 0].double() / stats[:, 2].double()).float()
    spread = (stats[:, 1].double() / stats[:, 2].double()).float() - score * score
    spread = torch.where(held, spread.clamp(min=0.0), math.inf)
    scope = torch.minimum(torch.minimum(torch.full_like(most, case["scope"]), most) + evict[:, 0] - 1, n)[:, None]
    inside = (_rank(spread) < scope) & held
    victim = (_rank(torch.where(inside, score, math.inf)) < evict) & held
    taken = victim | (~held & (slot < n_new[:, None]))
    # the tokens go to the taken slots in order
    order = (~taken).long().argsort(dim=1, stable=True)[:, :C]
    real_u = k < c[:, None]
    was = held.gather(1, order) & real_u
    there = lambda t: torch.where(was, t, -1).to(torch.int32).view(R, H, C).transpose(1, 2)[real]  # noqa: E731
    evicted_slot, evicted_pos = there(order), there(pos.gather(1, order))
    # probabilities of the chunk's rows, the mean of their heads
    lse = s["lse"][at].view(R, C, H, -1).permute(0, 2, 1, 3)
    p = torch.exp(_logits(s, 0, R) - lse[..., None]).mean(3).flatten(0, 1) * real_u[:, :, None]  # [units, C, B + C]
    sums, squares = p.sum(1), (p * p).sum(1)
    keep = (held & ~taken)[:, None, :]
    more = torch.stack([sums[:, :B], squares[:, :B], c[:, None].expand(-1, B).float()], 1)
    fresh = torch.stack([sums[:, B:], squares[:, B:], (c[:, None] - k).float()], 1)
    stats.copy_(torch.where(keep, stats + more, torch.where(taken[:, None, :], 0.0, stats)))
    at_unit, at_k = real_u.nonzero(as_tuple=True)
    at_slot, at_row = order[at_unit, at_k], at[r[at_unit], at_k]
    stats[at_unit, :, at_slot] = fresh[at_unit, :, at_k]
    pos[at_unit, at_slot] = s["qpos0"][r[at_unit]] + at_k.to(torch.int32)
    n_used.copy_(n_new)
    for cache, rows in ((s["K"], s["k_new"]), (s["V"], s["v_new"])):
        if "table" in s:
            cache[s["table"][r[at_unit], at_slot // s["page"]].long(), at_unit % H, at_slot % s["page"]] = rows[at_row, at_unit % H]
        else:
            cache[at_unit, at_slot] = rows[at_row, at_unit % H]
    return _committed(s, evicted_slot, evicted_pos)


def _committed(s, evicted_slot, evicted_pos):
    """What a commit leaves; the planes of the statistics are values of different kinds."""
    acc, acc2, count = s["stats"].unbind(1)
    return {"K": s["K"], "V": s["V"], "acc": acc, "acc2": acc2, "count": count, "pos": s["pos"], "n_used": s["n_used"],
            "evicted_slot": evicted_slot, "evicted_pos": evicted_pos}


def _plain_verify(s):
    """The requests side by side, the nodes in their order: a node's parent is decided before it."""
    case = s["case"]
    R, T, V = case["requests"], case["nodes"], case["vocab"]
    p, q, given, distinct = s["p"], s["q"], s["q"] is None, case["drafts"] == "distinct"
    r = torch.arange(R, device="cuda")
    parent = torch.arange(-1, T - 1, device="cuda").expand(R, T) if s["parent"] is None else s["parent"].long()
    tokens = s["tokens"].long()
    at = torch.zeros(R, dtype=torch.int64, device="cuda")                           # the last accepted node
    path, length = torch.zeros((R, T), dtype=torch.int64, device="cuda"), (s["n_nodes"] > 0).long()
    times, left, gone = (torch.full((R,), v, dtype=torch.float64, device="cuda") for v in (0.0, 1.0, 0.0))
    target = p[r, at].double()
    draft = torch.zeros_like(target) if given else q[r, at].double()
    for i in range(1, T):
        asked = (parent[:, i] == at) & (i < s["n_nodes"])
        x = tokens[:, i]
        pr, qr = target[r, x], draft[r, x]
        u = s["accept"][:, i].double()
        good = u * left < pr if given else u * qr * left < (pr - times * qr).clamp(min=0) * (1 - gone)
        yes, no = asked & good, asked & ~good
        if given:
            left = torch.where(no, left - pr, left)
            target[r, x] = torch.where(no, 0.0, pr)
        else:
            no = no & (gone < 1)  # (the earlier ones may hold all of the draft's distribution, by its roundings: then it has no other)
            times = torch.where(no, times + left / (1 - gone), times)
            gone = torch.where(no & distinct, gone + qr, gone)
            left = torch.where(no, (target - times[:, None] * draft).clamp(min=0).sum(1), left)
        at = torch.where(yes, i, at)
        path[r, length.clamp(max=T - 1)] = torch.where(yes, i, path[r, length.clamp(max=T - 1)])
        length = length + yes
        times, left, gone = torch.where(yes, 0.0, times), torch.where(yes, 1.0, left), torch.where(yes, 0.0, gone)
        target = torch.where(yes[:, None], p[r, at].double(), target)
        if not given:
            draft = torch.where(yes[:, None], q[r, at].double(), draft)
    weights = (target - times[:, None] * draft).clamp(min=0)
    weights = torch.where(weights.sum(1, keepdim=True) > 0, weights, p[r, at].double())
    sums = weights.cumsum(1)
    chosen = (sums > s["choose"].double()[:, None] * sums[:, -1:]).int().argmax(1)
    chosen = torch.where(length > 0, chosen, -1)
    return torch.where(torch.arange(T, device="cuda") < length[:, None], path, -1).int(), length.int(), chosen.int()


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if not own:
        return {"attend": _plain_attend, "commit": _plain_commit, "verify": _plain_verify}[case["op"]](s)
    import paper_2402_06262_amd as roco
    if case["op"] == "verify":
        roco.roco_tree_verify(s["p"], s["q"], s["tokens"], s["parent"], s["n_nodes"], s["accept"], s["choose"], s["path"], s["n_path"], s["next"],
                              s["workspace"], distinct=case["drafts"] == "distinct")
        return s["path"], s["n_path"], s["next"]
    if case["op"] == "attend":
        roco.roco_chunk_attend(s["params"], case["heads"], case["group"], s["pages"], s["q"], s["k_new"], s["v_new"], s["start"], s["qpos0"], s["K"],
                               s["V"], s["pos"], s["n_used"], s["out"], s["out_lse"], s["workspace"])
        return s["out"], s["out_lse"]
    s["state"].copy_(s["before"])
    roco.roco_chunk_commit(s["params"], case["heads"], case["group"], s["pages"], s["q"], s["k_new"], s["v_new"], s["lse"], s["start"], s["qpos0"],
                           s["K"], s["V"], s["stats"], s["pos"], s["n_used"], s["evicted_slot"], s["evicted_pos"], s["workspace"])
    return _committed(s, s["evicted_slot"], s["evicted_pos"])


def work(case):
    if case["op"] == "verify":
        # a row of the target's probabilities for each request, and of the draft's
        e = 2 if case["dtype"] == "bf16" else 4
        R, T, V = case["requests"], case["nodes"], case["vocab"]
        return {"bytes": float(R * (V * e * (1 if case["drafts"] == "given" else 2) + T * 24)), "flops": 3.0 * R * V}
    e = 2 if case["dtype"] == "bf16" else 4
    H, G, d = case["heads"], case["group"], case["head_dim"]
    _, used, tokens = _lengths(case)
    slots, total = float(H * sum(u for u, t in zip(used, tokens) if t)), sum(tokens)
    seen = float(H * G * sum(t * u + t * (t + 1) / 2 for u, t in zip(used, tokens)))
    if case["op"] == "attend":
        return {"bytes": slots * 2 * d * e + 2 * total * H * G * d * e + 4 * total * H * G + 2 * total * H * d * e + (4 * slots if case["window"] else 0),
                "flops": 4 * seen * d}
    return {"bytes": slots * (d * e + 24) + total * H * (G * d * e + 4 * G + 4 * d * e + 24), "flops": 2 * seen * d}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _exact_rows(s, cache, u, n):
    """The first n rows of unit u."""
    if "table" not in s:
        return cache[u, :n].double()
    H, page = s["case"]["heads"], s["page"]
    pages = s["table"][u // H, :-(-n // page)].long()
    return cache[pages, u % H].reshape(-1, cache.shape[-1])[:n].double()


def _exact_unit(s, u, n, a, b, first):
    """Logits of the tokens a .. b - 1 of the packed rows over the n slots of unit u and these tokens, [tokens, group, n + tokens]."""
    case = s["case"]
    H, G, w, c = case["heads"], case["group"], case["window"], b - a
    h = u % H
    keys = torch.cat([_exact_rows(s, s["K"], u, n), s["k_new"][a:b, h].double()])
    x = (s["q"][a:b, h * G:(h + 1) * G].double().reshape(c * G, -1) @ keys.t()).view(c, G, n + c) / math.sqrt(case["head_dim"])
    mine = first + torch.arange(c, device="cuda")
    if w:
        gap = mine[:, None] - torch.cat([s["pos"][u, :n].long(), mine])
        x += s["bias"] * ((gap >= 0) & (gap < w))[:, None, :]
    x[:, :, n:].masked_fill_(torch.ones((c, c), dtype=torch.bool, device="cuda").triu(1)[:, None, :], -math.inf)
    return x


def _exact_attend(s):
    case = s["case"]
    H, G, d = case["heads"], case["group"], case["head_dim"]
    total = len(s["q"])
    out = torch.zeros((total, H * G, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((total, H * G), dtype=torch.float64, device="cuda")
    start, used, first = s["start"].tolist(), s["n_used"].tolist(), s["qpos0"].tolist()
    for u, n in enumerate(used):
        r, h = divmod(u, H)
        a, b = start[r], start[r + 1]
        if a == b:
            continue
        x = _exact_unit(s, u, n, a, b, first[r])
        z = torch.logsumexp(x, -1)
        values = torch.cat([_exact_rows(s, s["V"], u, n), s["v_new"][a:b, h].double()])
        out[a:b, h * G:(h + 1) * G] = (torch.exp(x - z[..., None]).flatten(0, 1) @ values).view(b - a, G, d)
        lse[a:b, h * G:(h + 1) * G] = z
    return out, lse


def _exact_commit(s):
    case = s["case"]
    H, B, G = case["heads"], case["budget"], case["group"]
    result = s["stats"].double()
    start, used, first, budgets = s["start"].tolist(), s["n_used"].tolist(), s["qpos0"].tolist(), s["budget"].tolist()
    for u, n in enumerate(used):
        r, h = divmod(u, H)
        a, b = start[r], start[r + 1]
        c = b - a
        if c == 0:
            continue
        n_new = min(budgets[r], n + c)
        E = n + c - n_new
        slots = torch.arange(n, n_new, device="cuda")
        if E:
            acc, acc2, count = s["stats"][u, :, :n].cpu().unbind(0)  # (the choice is defined on 32-bit keys)
            score = acc / count
            spread = (acc2 / count - score * score).clamp(min=0)
            scope = spread.argsort(stable=True)[:min(n, min(case["scope"], budgets[r]) + E - 1)].sort().values
            victims = scope[score[scope].argsort(stable=True)[:E]].sort().values
            slots = torch.cat([victims.cuda(), slots])
        x = _exact_unit(s, u, n, a, b, first[r])
        p = torch.exp(x - s["lse"][a:b, h * G:(h + 1) * G].double()[..., None]).mean(1)
        sums = torch.stack([p.sum(0), (p * p).sum(0)])
        result[u, :2, :n] += sums[:, :n]
        result[u, 2, :n] += c
        result[u, :2, slots] = sums[:, n:]
        result[u, 2, slots] = (c - torch.arange(c, device="cuda")).double()
    acc, acc2, count = result.unbind(1)
    return {"K": None, "V": None, "acc": acc, "acc2": acc2, "count": count, "pos": None, "n_used": None, "evicted_slot": None,
            "evicted_pos": None}


def exact(case, seed):
    if case["op"] == "verify":
        return None  # whole numbers
    s = prepare(case, seed)
    return _exact_attend(s) if case["op"] == "attend" else _exact_commit(s)
