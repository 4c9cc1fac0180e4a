"""Verification of drafted trees (roco_tree_verify) against the float64 oracle, which forms every distribution literally: whole numbers, equal."""
import numpy as np
import pytest
import torch

import paper_2402_06262_amd as roco
from oracle.verify import tree_verify

pytestmark = pytest.mark.gpu


class Batch:
    def __init__(self, seed, R, T, V, children=1, drafts="sampled", dtype="f32", n_nodes=None, spread=2.0, apart=1.0, pad=0):
        rng = np.random.default_rng(seed)
        self.R, self.T, self.V, self.drafts, self.chain = R, T, V, drafts, children == 1
        logits = spread * rng.standard_normal((R, T, V))
        soft = lambda x: np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True)  # noqa: E731
        p = soft(logits)
        p = p * (p > 1e-3 * p.max(-1, keepdims=True))
        q = soft(logits + apart * rng.standard_normal((R, T, V)))
        tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        # rows with a stride of their own
        as_rows = lambda x: torch.nn.functional.pad(torch.from_numpy(x).float(), (0, pad)).to(tdt).cuda()[..., :V]  # noqa: E731
        self.p, self.q = as_rows(p / p.sum(-1, keepdims=True)), as_rows(q)
        self.hp, self.hq = self.p.double().cpu().numpy(), self.q.double().cpu().numpy()
        self.parent = np.array([[-1] + [i - 1 if self.chain else max(0, (i - 1) // children - int(rng.integers(0, 2))) for i in range(1, T)] for _ in range(R)])
        self.tokens = np.zeros((R, T), np.int64)
        for r in range(R):
            for j in range(T):
                kids = np.flatnonzero(self.parent[r] == j)
                if len(kids):
                    w = self.hq[r, j] / self.hq[r, j].sum()
                    if drafts == "sampled":
                        self.tokens[r, kids] = rng.choice(V, len(kids), p=w)
                    else:
                        order = np.argsort(-(w + 1e-300) / rng.exponential(size=V))
                        self.tokens[r, kids] = np.resize(order[:V], len(kids))
        self.n_nodes = np.full(R, T) if n_nodes is None else np.array(n_nodes)
        self.accept, self.choose = rng.random((R, T), dtype=np.float32), rng.random(R, dtype=np.float32)

    def run(self, max_path=None, **kw):
        i = lambda x: torch.from_numpy(np.ascontiguousarray(x)).int().cuda()  # noqa: E731
        f = lambda x: torch.from_numpy(np.ascontiguousarray(x)).float().cuda()  # noqa: E731
        self.max_path = max_path or self.T
        path = torch.full((self.R, self.max_path), -9, dtype=torch.int32, device="cuda")
        n_path, nxt = (torch.full((self.R,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
        ws = torch.full((roco.verify_workspace_bytes(self.R, self.T, self.V),), 0xEE, dtype=torch.uint8, device="cuda")
        a = dict(p=self.p, q=None if self.drafts == "given" else self.q, tokens=i(self.tokens), parent=None if self.chain else i(self.parent), n_nodes=i(self.n_nodes),
                 accept=f(self.accept), choose=f(self.choose), path=path, n_path=n_path, next_token=nxt, workspace=ws, distinct=self.drafts == "distinct")
        a.update(kw)
        roco.roco_tree_verify(**a)
        torch.cuda.synchronize()
        return path.cpu().numpy(), n_path.cpu().numpy(), nxt.cpu().numpy()

    def check(self, path, n_path, nxt):
        for r in range(self.R):
            want, token = tree_verify(self.hp[r], None if self.drafts == "given" else self.hq[r], self.tokens[r], None if self.chain else self.parent[r],
                                      int(self.n_nodes[r]), self.accept[r], self.choose[r], self.drafts == "distinct", self.max_path)
            assert n_path[r] == len(want) and path[r].tolist() == want + [-1] * (self.max_path - len(want)), f"request {r}"
            assert nxt[r] == token, f"request {r}: token"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drafts", ["sampled", "distinct", "given"])
@pytest.mark.parametrize("R,T,V,children", [(1, 1, 1, 1), (3, 1, 700, 1), (5, 4, 7, 1), (6, 9, 1000, 1), (4, 64, 333, 1), (5, 12, 2051, 2), (7, 33, 515, 3), (3, 64, 4100, 5),
                                            (2, 40, 90, 39)])
def test_trees(dtype, drafts, R, T, V, children):
    b = Batch(R + T + V, R, T, V, children, drafts, dtype)
    b.check(*b.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 1, 3, 8])
def test_rows_of_any_alignment(dtype, pad):
    b = Batch(pad, 5, 7, 4099, 2, "sampled", dtype, pad=pad)
    b.check(*b.run())
    # q's rows lie differently from those of p
    q = torch.nn.functional.pad(b.q, (0, 5))[..., :b.V]
    b.check(*b.run(q=q))


@pytest.mark.parametrize("rounds", [1, 2, 4])
def test_rounds(rounds, monkeypatch):
    monkeypatch.setenv("ROCO_VERIFY_ROUNDS", str(rounds))
    b = Batch(rounds, 6, 40, 3000, 6, "distinct", apart=2.5)
    b.check(*b.run())


@pytest.mark.parametrize("max_path", [1, 2, 5])
def test_short_paths_and_sizes_of_trees(max_path):
    b = Batch(max_path, 9, 16, 500, 2, n_nodes=[0, 1, 2, 3, 16, 15, 8, 0, 16], apart=0.1)
    b.check(*b.run(max_path=max_path))


def test_large_vocabulary():
    b = Batch(5, 3, 6, 131072, 2, "distinct", spread=4.0)
    b.check(*b.run())


@pytest.mark.parametrize("drafts", ["sampled", "distinct", "given"])
@pytest.mark.parametrize("bad", [np.nan, -0.25, -np.inf])
def test_what_is_no_probability_counts_as_zero(drafts, bad):
    b = Batch(11, 8, 9, 300, 3, drafts, apart=1.5)
    for t in (b.p, b.q):
        t[:, :, 5::7] = bad
    b.tokens[:, 3::4] = 12  # (one of those)
    b.hp, b.hq = b.p.double().cpu().numpy(), b.q.double().cpu().numpy()
    b.check(*b.run())
    b.p[2:4] = bad  # nothing is left at all
    b.hp = b.p.double().cpu().numpy()
    path, n_path, nxt = b.run()
    b.check(path, n_path, nxt)
    assert (nxt[2:4] == -1).all()


def test_tokens_outside_the_vocabulary_and_parents_that_are_none():
    b = Batch(12, 4, 8, 200, 2, "sampled", apart=0.1)
    b.tokens[0, 1], b.tokens[1, 1], b.tokens[2, 2] = -1, 200, 2 ** 31 - 1
    b.parent[0, 2], b.parent[1, 3], b.parent[3, 4] = 5, -3, 4
    b.check(*b.run())


@pytest.mark.parametrize("value", [0.0, 1.0 - 2.0 ** -24])
def test_random_numbers_at_the_ends(value):
    for drafts in ("sampled", "distinct", "given"):
        b = Batch(13, 5, 7, 5000, 2, drafts)
        b.accept[:], b.choose[:] = value, value
        b.check(*b.run())


def test_accepted_whole_where_draft_and_target_agree():
    b = Batch(14, 6, 8, 1000, 1, apart=0.0)
    b.q = b.p.clone()
    b.hq = b.hp
    for r in range(6):
        b.tokens[r, 1:] = [np.argmax(b.hp[r, i]) for i in range(7)]
    path, n_path, nxt = b.run()
    b.check(path, n_path, nxt)
    assert (n_path == 8).all()


def test_requests_that_share_rows_of_the_draft():
    b = Batch(15, 6, 5, 800, 2)
    shared = b.q[:1].expand(6, -1, -1)
    b.hq = shared.double().cpu().numpy()
    b.check(*b.run(q=shared))


def test_many_requests():
    b = Batch(16, 700, 3, 64, 2, "distinct")
    b.check(*b.run())


def test_as_many_requests_as_a_call_has():
    b = Batch(20, 65535, 2, 5, 1)
    b.check(*b.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 3])
def test_the_largest_vocabulary(dtype, pad):
    """2^22 tokens, the borders' last ones among those that are chosen."""
    b = Batch(21, 3, 2, 1 << 22, 1, dtype=dtype, pad=pad, apart=3.0)
    b.choose[:] = [1.0 - 2.0 ** -24, 0.0, 0.5]
    b.check(*b.run())


def test_captured_and_replayed_with_other_inputs():
    """Graphs of two shapes that share a workspace; a pass leaves nothing for the next."""
    batches = [Batch(17, 5, 12, 9000, 3, "distinct"), Batch(18, 9, 5, 3000, 1)]
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x)).float().cuda()  # noqa: E731
    ws = torch.full((max(roco.verify_workspace_bytes(b.R, b.T, b.V) for b in batches),), 0xEE, dtype=torch.uint8, device="cuda")
    side, graphs = torch.cuda.Stream(), []
    for b in batches:
        b.max_path = b.T
        i = lambda x: torch.from_numpy(np.ascontiguousarray(x)).int().cuda()  # noqa: E731
        b.out = [torch.full((b.R, b.T), -9, dtype=torch.int32, device="cuda")] + [torch.full((b.R,), -9, dtype=torch.int32, device="cuda") for _ in range(2)]
        b.numbers = f(b.accept), f(b.choose)
        args = (b.p, b.q, i(b.tokens), None if b.chain else i(b.parent), i(b.n_nodes), *b.numbers, *b.out, ws)
        b.call = lambda b=b, args=args: roco.roco_tree_verify(*args, distinct=b.drafts == "distinct")
        b.call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            b.call()
        graphs.append(graph)
    rng = np.random.default_rng(0)
    for turn in range(4):
        for b, graph in zip(batches, graphs):
            b.accept, b.choose = rng.random((b.R, b.T), dtype=np.float32), rng.random(b.R, dtype=np.float32)
            for t, x in zip(b.numbers, (b.accept, b.choose)):
                t.copy_(f(x))
            torch.cuda.synchronize()
            if turn == 2:
                b.call()
            else:
                graph.replay()
            torch.cuda.synchronize()
            b.check(*(t.cpu().numpy() for t in b.out))


def test_rows_beyond_32_bits_of_elements():
    """The last request's rows begin behind 2^32 bytes."""
    R, T = 3, 2
    b = Batch(19, R, T, 500, 1)
    far = torch.zeros((R, (1 << 29) + 64), device="cuda")
    p = far.as_strided((R, T, 500), (far.stride(0), 600, 1))
    p.copy_(b.p)
    assert p.stride(0) * (R - 1) * 4 > 1 << 32
    b.check(*b.run(p=p))
