"""Chunks of new tokens over budgeted caches (roco_chunk_attend, roco_chunk_commit) against the float64 oracle, element by element: a chunk is a
drafted chain of any length (oracle/trees.py).

Tolerances, from the roundings of the two storage types and of fp32 (u = 2^-24):
  logits   a product of d terms in fp32, scaled: within x = (d + 8) u L, L the row's largest scale sum |q k|; 2^x then moves a probability by a
           factor of x (natural logarithm), the exponential's and the sum's own roundings by (8 + sqrt of the number of terms) u
  outputs  rel = 2 x + (8 + 2 sqrt n) u of sum p |v|; probabilities of bf16 are one bf16 number each, half a step of 2^-8 off, and their sum, which
           divides, is that of the unrounded ones: 2^-8 of sum p |v| more; half a step of the type
  lse      x + (8 + sqrt n) u + 2^-22 |lse|
  Acc      what a chunk adds: 2 x + (8 + sqrt of its rows) u of it, and half a step of the sum; Acc2 twice that
"""
import math

import numpy as np
import pytest
import torch

import paper_2402_06262_amd as roco
from inputs import round_to_bf16
from oracle import roco_oracle as orc
from oracle import trees

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_IMPORTANCE = {"mas": 0, "aas": 1, "oldest": 2, "ltas": 3, "aqas": 4}
_SCOPE = {"std": 0, "window": 1, "all": 2}


def dev(x, dtype=None):
    x = torch.from_numpy(np.ascontiguousarray(x))
    return (x.to(torch.int32) if dtype is None else x.float().to(_DT[dtype])).cuda()


class Step:
    """A step's inputs on the host, and on the device on demand: `requests` x `heads` units of their own fills, and a chunk for each request.  spare: rows
    of the packed arrays before the first request's and behind the last one's; fused: q, k and v in one array."""

    def __init__(self, seed, dtype, d, used, tokens, heads=2, group=1, B=None, page=0, budgets=None, window=0, bias=0.75, scope=8, policy=None, spare=(0, 0),
                 fused=True, n_extra=3):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.d, self.heads, self.group, self.page, self.window, self.scope = rng, dtype, d, heads, group, page, window, scope
        self.R = R = len(used)
        self.U = R * heads
        self.B = B = B or max(max(used), 1)
        self.budgets = budgets or [B] * R
        self.used, self.tokens = used, tokens
        self.start = [spare[0]]
        for t in tokens:
            self.start.append(self.start[-1] + t)
        self.total = self.start[-1] + spare[1]
        self.policy, self.sc, self.bias, self.fused = policy, 1 / math.sqrt(d), bias if window else 0.0, fused
        rnd = round_to_bf16 if dtype == "bf16" else (lambda x: x)
        draw = lambda *s: rnd(rng.standard_normal(s).astype(np.float32))  # noqa: E731
        self.K, self.V = draw(self.U, B, d), draw(self.U, B, d)
        self.q, self.k_new, self.v_new = draw(self.total, heads * group, d), draw(self.total, heads, d), draw(self.total, heads, d)
        self.qpos0 = rng.integers(B + 5, B + 50, R)
        self.pos = np.full((self.U, B), -1)
        self.stats = np.zeros((self.U, 3, B), np.float32)
        for u in range(self.U):
            n = used[u // heads]
            self.pos[u, :n] = self.qpos0[u // heads] - 1 - rng.permutation(n)
            c = rng.integers(1, 400, n)
            m = np.exp(rng.standard_normal(n)) / B
            self.stats[u, 0, :n], self.stats[u, 2, :n] = m * c, c
            self.stats[u, 1, :n] = (m ** 2 * (1 + np.exp(rng.standard_normal(n)))) * c
        if page:
            need = [-(-b // page) for b in self.budgets]
            self.M = -(-B // page)
            self.n_pages = sum(need) + n_extra
            order = rng.permutation(self.n_pages).tolist()
            self.table = np.array([[order.pop() if j < k else -1 for j in range(self.M)] for k in need])

    def upload(self):
        f, i = (lambda x: dev(x, self.dtype)), dev
        self.p = roco.RocoParams(self.U, self.d, self.B, min(self.scope, self.B), roco.ROCO_BF16 if self.dtype == "bf16" else roco.ROCO_F32, 0.0,
                                 self.window, self.bias, *((_IMPORTANCE[self.policy.importance], _SCOPE[self.policy.scope_kind], self.policy.sinks)
                                                           if self.policy else ()))
        H, G = self.heads, self.group
        if self.fused:
            qkv = f(np.concatenate([self.q, self.k_new, self.v_new], 1))
            self.dq, self.dk, self.dv = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
        else:
            self.dq, self.dk, self.dv = f(self.q), f(self.k_new), f(self.v_new)
        self.dstart, self.dqpos0, self.dpos = i(np.array(self.start)), i(self.qpos0), i(self.pos)
        self.dn_used = i(np.repeat(self.used, H))
        self.dstats = torch.from_numpy(self.stats).cuda()
        if self.page:
            self.dK, self.dV = f(self.pool(self.K)), f(self.pool(self.V))
            self.pages = roco.RocoPages(i(self.table), self.n_pages, self.page, i(np.array(self.budgets)))
        else:
            self.dK, self.dV, self.pages = f(self.K), f(self.V), None
        self.ws = torch.empty(roco.chunk_workspace_bytes(self.p, H, G, self.total), dtype=torch.uint8, device="cuda").fill_(0xEE)
        self.out = torch.full((self.total, H * G, self.d), 77.0, dtype=_DT[self.dtype], device="cuda")
        self.lse = torch.full((self.total, H * G), 77.0, device="cuda")
        return self

    def pool(self, rows, fill=np.nan):
        """[n_pages, heads, page, d]; what no slot in use names is NaN."""
        pool = np.full((self.n_pages, self.heads, self.page, self.d), fill, np.float32)
        for u in range(self.U):
            r, h = divmod(u, self.heads)
            for j in range(self.used[r]):
                e = self.table[r, j // self.page]
                if 0 <= e < self.n_pages:
                    pool[e, h, j % self.page] = rows[u, j]
        return pool

    def unpool(self, pool, u, n):
        r, h = divmod(u, self.heads)
        return np.stack([pool[self.table[r, j // self.page], h, j % self.page] for j in range(n)]) if n else np.zeros((0, self.d), np.float32)

    def attend(self, **kw):
        a = dict(pages=self.pages, q=self.dq, k_new=self.dk, v_new=self.dv, token_start=self.dstart, qpos0=self.dqpos0, K_cache=self.dK, V_cache=self.dV,
                 pos=self.dpos, n_used=self.dn_used, out=self.out, lse=self.lse, workspace=self.ws)
        a.update(kw)
        roco.roco_chunk_attend(self.p, self.heads, self.group, **a)
        torch.cuda.synchronize()
        return self.out.float().cpu().numpy().astype(np.float64), self.lse.cpu().numpy().astype(np.float64)

    def rows(self, u):
        """(query rows, keys, values) of the unit's chunk."""
        r, h = divmod(u, self.heads)
        a, b, G = self.start[r], self.start[r + 1], self.group
        return self.q[a:b, h * G:(h + 1) * G], self.k_new[a:b, h], self.v_new[a:b, h]

    def want(self, u):
        r = u // self.heads
        n = self.used[r]
        q, k, v = self.rows(u)
        return trees.tree_attend(self.K[u, :n], self.V[u, :n], self.pos[u], q, k, v, list(range(-1, self.tokens[r] - 1)), int(self.qpos0[r]), self.sc,
                                 self.window, self.bias)

    def check_attend(self, out, lse, what="", units=None):
        spare = np.ones(self.total, bool)
        spare[self.start[0]:self.start[-1]] = False
        assert (out[spare] == 77).all() and (lse[spare] == 77).all(), f"{what}: rows that are no request's"
        for u in range(self.U) if units is None else units:
            r, h = divmod(u, self.heads)
            if self.tokens[r] == 0:
                continue
            a, b, heads = self.start[r], self.start[r + 1], slice(h * self.group, (h + 1) * self.group)
            w = self.want(u)
            n = self.used[r] + self.tokens[r]
            x = (self.d + 8) * U * w.logit
            rel = 2 * x + (8 + 2 * math.sqrt(n)) * U + (0 if self.dtype == "f32" else 2.0 ** -8)
            half = 2.0 ** -8 if self.dtype == "bf16" else U
            err = np.abs(out[a:b, heads] - w.out)
            tol = rel * w.mass + half * np.abs(w.out) + 1e-30
            assert (err <= tol).all(), f"{what} unit {u}: outputs, worst {np.nanmax(err / tol):.3g} of the tolerance, {np.isnan(err).sum()} NaN"
            err = np.abs(lse[a:b, heads] - w.lse)
            tol = x + (8 + math.sqrt(n)) * U + 2.0 ** -22 * np.abs(w.lse)
            assert (err <= tol).all(), f"{what} unit {u}: lse, worst {np.nanmax(err / tol):.3g} of the tolerance"

    def exact_lse(self):
        """The normalisers by the oracle, rounded to fp32: the step under test is then the commit alone."""
        lse = np.full((self.total, self.heads * self.group), 55.0, np.float32)
        for u in range(self.U):
            r, h = divmod(u, self.heads)
            if self.tokens[r]:
                lse[self.start[r]:self.start[r + 1], h * self.group:(h + 1) * self.group] = self.want(u).lse
        return lse

    def commit(self, host_lse, **kw):
        self.ev_slot = torch.full((self.total, self.heads), -7, dtype=torch.int32, device="cuda")
        self.ev_pos = torch.full((self.total, self.heads), -7, dtype=torch.int32, device="cuda")
        a = dict(pages=self.pages, q=self.dq, k_new=self.dk, v_new=self.dv, lse=dev(host_lse, "f32"), token_start=self.dstart, qpos0=self.dqpos0,
                 K_cache=self.dK, V_cache=self.dV, stats=self.dstats, pos=self.dpos, n_used=self.dn_used, evicted_slot=self.ev_slot, evicted_pos=self.ev_pos,
                 workspace=self.ws)
        a.update(kw)
        roco.roco_chunk_commit(self.p, self.heads, self.group, **a)
        torch.cuda.synchronize()

    def check_commit(self, lse, what=""):
        ev_slot, ev_pos = self.ev_slot.cpu().numpy(), self.ev_pos.cpu().numpy()
        stats, pos, used = self.dstats.cpu().numpy().astype(np.float64), self.dpos.cpu().numpy(), self.dn_used.cpu().numpy()
        K, V = self.dK.float().cpu().numpy(), self.dV.float().cpu().numpy()
        spare = np.ones(self.total, bool)
        spare[self.start[0]:self.start[-1]] = False
        assert (ev_slot[spare] == -7).all() and (ev_pos[spare] == -7).all(), f"{what}: rows that are no request's"
        for u in range(self.U):
            r, h = divmod(u, self.heads)
            n, c = self.used[r], min(self.tokens[r], self.budgets[r])
            st = orc.CacheState(self.K[u].astype(np.float64), self.V[u].astype(np.float64), *self.stats[u].astype(np.float64), self.pos[u].copy(), n)
            before = self.stats[u].astype(np.float64)
            q, k, v = self.rows(u)
            a, b = self.start[r], self.start[r + 1]
            z = lse[a:b, h * self.group:(h + 1) * self.group]
            t = trees.tree_commit(st, self.budgets[r], q, k, v, z, list(range(c)), int(self.qpos0[r]), min(self.scope, self.B), self.sc, self.window, self.bias,
                                  self.policy)
            w = f"{what} unit {u}"
            assert ev_slot[a:a + c, h].tolist() == t.evicted_slot.tolist() and (ev_slot[a + c:b, h] == -1).all(), w
            assert ev_pos[a:a + c, h].tolist() == t.evicted_pos.tolist() and (ev_pos[a + c:b, h] == -1).all(), w
            assert used[u] == st.n_used and (pos[u] == st.pos).all(), w
            m = st.n_used
            for got, want, name in ((K, st.K, "K"), (V, st.V, "V")):
                rows = self.unpool(got, u, m) if self.page else got[u, :m]
                assert (rows == want[:m]).all(), f"{w}: {name}"
            assert (stats[u, 2] == st.count).all(), w
            assert (stats[u, :2, m:] == before[:2, m:]).all(), f"{w}: slots that are not in use"
            if c == 0:
                assert (stats[u] == before).all(), w
                continue
            x = (self.d + 8) * U * self.sc * self.d * max(np.abs(self.K).max(), np.abs(self.k_new).max()) * np.abs(q).max()  # above every row's
            rel = 2 * x + (8 + math.sqrt(c * self.group)) * U
            err = np.abs(stats[u, 0, :m] - st.acc[:m])
            tol = rel * t.mass[0, :m] + 2 * U * np.abs(st.acc[:m]) + 1e-30
            assert (err <= tol).all(), f"{w}: Acc, worst {np.nanmax(err / tol):.3g} of the tolerance"
            err = np.abs(stats[u, 1, :m] - st.acc2[:m])
            tol = 2 * rel * (t.mass[0, :m] if self.policy and self.policy.importance == "ltas" else t.mass[1, :m]) + 2 * U * np.abs(st.acc2[:m]) + 1e-30
            if self.policy and self.policy.importance == "aqas":
                tol = tol + near_average(self, u, q[:c], z[:c], st)
            assert (err <= tol).all(), f"{w}: Acc2, worst {np.nanmax(err / tol):.3g} of the tolerance"


def near_average(s, u, q, lse, st):
    """How many of the chunk's rows give a slot a probability so near their average that fp32 may count it or not."""
    m, n = st.n_used, s.used[u // s.heads]
    near = np.zeros(m)
    for k in range(len(q)):
        p = np.exp(q[k].astype(np.float64) @ st.K[:m].T * s.sc - lse[k][:, None]).mean(0)
        near += np.abs(p * (n + k + 1) - 1) < 1e-4
    return near


# ---------------------------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("used,tokens,group", [
    ([1], [1], 1), ([0], [1], 1), ([0], [33], 1), ([31, 32, 33], [1, 0, 2], 1), ([64, 0, 500], [5, 130, 1], 3), ([100, 7], [129, 257], 1), ([257], [200], 4),
    ([40, 300, 0, 5], [1, 1, 1, 1], 8), ([90], [40], 7), ([65, 200], [3, 17], 64)])
def test_attention(dtype, d, used, tokens, group):
    s = Step(7 * len(used) + d + sum(tokens), dtype, d, used, tokens, group=group, B=max(used) + 3, spare=(2, 3)).upload()
    s.check_attend(*s.attend())


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 1024])
def test_pages(dtype, d, page):
    s = Step(page + d, dtype, d, [200, 17, 0, 333, 16], [70, 1, 5, 150, 0], heads=3, group=2, page=page, budgets=[220, 40, 64, 400, 16], B=400).upload()
    s.check_attend(*s.attend())


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("window,page", [(1, 0), (20, 0), (300, 16), (100000, 64)])
def test_recency_windows(dtype, d, window, page):
    s = Step(window + d, dtype, d, [120, 33, 0], [50, 1, 40], group=3, window=window, page=page, B=200).upload()
    s.check_attend(*s.attend())


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_splits(dtype, d, splits, monkeypatch):
    monkeypatch.setenv("ROCO_CHUNK_SPLITS", str(splits))
    s = Step(splits + d, dtype, d, [500, 3, 0], [20, 130, 1], group=2, B=600, spare=(1, 2)).upload()
    s.check_attend(*s.attend())


@pytest.mark.parametrize("dtype,d", TYPES)
def test_rows_of_their_own(dtype, d):
    s = Step(d, dtype, d, [50, 10], [20, 3], group=2, fused=False).upload()
    s.check_attend(*s.attend())


@pytest.mark.parametrize("requests", [63, 64, 65, 130])
def test_many_requests(requests):
    rng = np.random.default_rng(requests)
    s = Step(requests, "bf16", 64, rng.integers(0, 60, requests).tolist(), rng.integers(0, 4, requests).tolist(), heads=1, group=40, B=64).upload()
    s.check_attend(*s.attend())


# ---------------------------------------------------------------------------------------------------- taking over
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("used,tokens,group,B", [
    ([1], [1], 1, 1), ([0], [1], 1, 4), ([50, 7, 0], [20, 1, 0], 1, 60), ([60, 60, 0], [7, 60, 33], 2, 60), ([300], [130], 4, 310), ([280, 100], [90, 200], 8, 300),
    ([90], [70], 3, 100), ([40, 200], [3, 90], 16, 200), ([40, 50], [9, 33], 17, 60), ([33], [20], 64, 40), ([5, 20], [50, 40], 5, 30)])
def test_commits(dtype, d, used, tokens, group, B):
    s = Step(3 * sum(used) + d + group, dtype, d, used, tokens, group=group, B=B, spare=(1, 2)).upload()
    lse = s.exact_lse()
    s.commit(lse)
    s.check_commit(lse)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page,window", [(16, 0), (64, 0), (32, 25)])
def test_paged_commits(dtype, d, page, window):
    s = Step(page + d, dtype, d, [200, 17, 0, 333, 16], [70, 30, 5, 150, 0], heads=3, group=2, page=page, window=window, budgets=[220, 40, 64, 333, 16], B=400).upload()
    lse = s.exact_lse()
    s.commit(lse)
    s.check_commit(lse)


@pytest.mark.parametrize("policy", [orc.Policy("aas", "std", 0), orc.Policy("oldest", "all", 4), orc.Policy("ltas", "all", 0), orc.Policy("aqas", "window", 0),
                                    orc.Policy("mas", "window", 0)], ids=lambda p: f"{p.importance}-{p.scope_kind}")
@pytest.mark.parametrize("group", [1, 3, 20])
def test_policies(policy, group):
    s = Step(group, "bf16", 128, [80, 20, 100], [30, 30, 10], group=group, B=100, policy=policy, scope=40).upload()
    lse = s.exact_lse()
    s.commit(lse)
    s.check_commit(lse)
