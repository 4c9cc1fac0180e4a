"""Refusals of the chunks' and the verification's entry points, all on the host (no GPU: nothing is launched), through the C ABI, the extension module and
ctypes alone."""
import ctypes

import pytest
import torch

import paper_2402_06262_amd as roco
from paper_2402_06262_amd import binding

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3
OK = 0x1000
P = roco.RocoParams(8, 128, 256, 16, roco.ROCO_BF16)


def _pages(n_pages=40, page=64, max_pages=4, table=OK, budget=None):
    return roco.RocoPages(table, n_pages, page, budget, max_pages)


def _attend(params=P, heads=4, group=2, tokens=100, pages=None, strides=(1024, 512), ws=None, ptrs=None, lse=OK):
    p = [OK] * 11 if ptrs is None else ptrs
    need = roco.chunk_workspace_bytes(P, 4, 2, 100) if ws is None else ws
    return roco.load_library().roco_chunk_attend(ctypes.byref(params), heads, group, tokens, None if pages is None else ctypes.byref(pages), p[0], strides[0], p[1], p[2],
                                              strides[1], p[3], p[4], p[5], p[6], p[7], p[8], p[9], lse, p[10], need, None)


def _commit(params=P, heads=4, group=2, tokens=100, pages=None, strides=(1024, 512), ws=None, ptrs=None, evicted=(OK, OK)):
    p = [OK] * 12 if ptrs is None else ptrs
    need = roco.chunk_workspace_bytes(P, 4, 2, 100) if ws is None else ws
    return roco.load_library().roco_chunk_commit(ctypes.byref(params), heads, group, tokens, None if pages is None else ctypes.byref(pages), p[0], strides[0], p[1],
                                                 p[2], strides[1], *p[3:11], *evicted, p[11], need, None)


@pytest.mark.parametrize("call", [_attend, _commit])
def test_shapes_are_checked(call):
    need = roco.chunk_workspace_bytes(P, 4, 2, 100)
    assert need > 0 and call(ws=0) == call(ws=need - 1) == EWORKSPACE  # everything else is in order
    assert call(heads=0) == EINVAL and call(heads=3) == EINVAL and call(heads=-4) == EINVAL  # 8 units
    assert call(group=0) == EINVAL and call(tokens=0) == EINVAL and call(tokens=-1) == EINVAL
    assert call(group=65, strides=(1 << 20, 512)) == EUNSUPPORTED
    assert call(tokens=1 << 28, ws=1 << 60) == EUNSUPPORTED  # 2^31 rows
    for kw, code in ((dict(units=0), EINVAL), (dict(scope=257), EINVAL), (dict(head_dim=96), EUNSUPPORTED), (dict(dtype=2), EUNSUPPORTED),
                     (dict(scale=float("nan")), EINVAL), (dict(recency_window=-1), EINVAL), (dict(units=65536), EUNSUPPORTED)):
        bad = roco.RocoParams(**{**dict(units=8, head_dim=128, budget=256, scope=16, dtype=roco.ROCO_BF16), **kw})
        assert call(bad, ws=1 << 40) == code
        assert roco.chunk_workspace_bytes(bad, 4, 2, 100) == 0
    assert call(roco.RocoParams(65532, 128, 1 << 17, 16, roco.ROCO_BF16), ws=1 << 50) == EUNSUPPORTED
    assert roco.chunk_workspace_bytes(P, 0, 2, 100) == roco.chunk_workspace_bytes(P, 4, 65, 100) == roco.chunk_workspace_bytes(P, 4, 2, 0) == 0


@pytest.mark.parametrize("call", [_attend, _commit])
def test_strides_are_checked(call):
    assert call(strides=(1032, 520), ws=0) == EWORKSPACE  # multiples of 16 bytes
    for strides in ((1016, 512), (1024, 504), (1028, 512), (1024, 516), (0, 512), (1024, -512)):
        assert call(strides=strides) == EINVAL
    assert call(strides=(1 << 23, 1 << 23), ws=0) == EWORKSPACE
    for strides in (((1 << 23) + 8, 512), (1024, (1 << 23) + 8)):
        assert call(strides=strides) == EUNSUPPORTED


@pytest.mark.parametrize("call", [_attend, _commit])
@pytest.mark.parametrize("dtype", [roco.ROCO_BF16, roco.ROCO_F32])
def test_strides_whose_bytes_pass_64_bits(call, dtype):
    """Distances of a token are bounded before they are counted in bytes: 2^62 elements of four bytes are 0 in 64 bits, and 2^62 + 2^20 an ordinary stride."""
    p = roco.RocoParams(8, 128, 256, 16, dtype)
    for far in (1 << 60, 1 << 61, 1 << 62, (1 << 62) + (1 << 20), (1 << 63) - (1 << 20), (1 << 63) - 8):
        for strides in ((far, 512), (1024, far)):
            assert call(p, strides=strides, ws=0) == EUNSUPPORTED, (far, strides)
    for far in ((1 << 63) - 1, (1 << 24) + 1):  # neither a multiple of 16 bytes nor near enough
        for strides in ((far, 512), (1024, far)):
            assert call(p, strides=strides, ws=0) in (EINVAL, EUNSUPPORTED), (far, strides)


@pytest.mark.parametrize("call", [_attend, _commit])
def test_pages_are_checked(call):
    assert call(pages=_pages(), ws=0) == EWORKSPACE
    assert call(pages=_pages(table=None)) == EINVAL and call(pages=_pages(table=OK + 2)) == EINVAL and call(pages=_pages(budget=OK + 2)) == EINVAL
    assert call(pages=_pages(table=OK + 4, budget=OK + 8), ws=0) == EWORKSPACE
    for page in (0, 8, 48, 2048, -16):
        assert call(pages=_pages(page=page, max_pages=1 << 20)) == EINVAL
    assert call(pages=_pages(max_pages=3)) == EINVAL  # 192 slots for a budget of 256
    assert call(pages=_pages(max_pages=0)) == EINVAL and call(pages=_pages(n_pages=0)) == EINVAL
    assert call(pages=_pages(n_pages=1 << 23)) == EUNSUPPORTED  # 2^31 rows


def test_pointers_are_checked():
    # rows and workspaces are aligned to 16 bytes, words to 4
    for call, n, words in ((_attend, 11, (3, 4, 7, 8)), (_commit, 12, (3, 4, 5, 8, 9, 10))):
        for i in range(n):
            assert call(ptrs=[OK + 4 if j == i else OK for j in range(n)], ws=0) == (EWORKSPACE if i in words else EINVAL), i
            for bad in (None, OK + (2 if i in words else 8)):
                assert call(ptrs=[bad if j == i else OK for j in range(n)]) == EINVAL, i
    assert _attend(lse=None, ws=0) == EWORKSPACE and _attend(lse=OK + 2, ws=1 << 40) == EINVAL
    assert _commit(evicted=(None, None), ws=0) == EWORKSPACE
    assert _commit(evicted=(OK + 2, OK), ws=1 << 40) == _commit(evicted=(OK, OK + 2), ws=1 << 40) == EINVAL


def test_workspaces_follow_the_choice_of_shares(monkeypatch):
    sizes = []
    for name, value in ((None, None), ("ROCO_CHUNK_SPLITS", "64"), ("ROCO_CHUNK_ROW_SPLITS", "16")):
        if name:
            monkeypatch.setenv(name, value)
        sizes.append(roco.chunk_workspace_bytes(P, 4, 2, 100))
    assert sizes[0] < sizes[1] <= sizes[2]


@pytest.mark.parametrize("env", [{}, {"ROCO_CHUNK_SPLITS": "7"}, {"ROCO_CHUNK_SPLITS": "1"}, {"ROCO_CHUNK_ROWS": "32"}, {"ROCO_CHUNK_ROWS": "128"}, {"ROCO_CHUNK_ROWS": "256"},
                                 {"ROCO_CHUNK_ROW_SPLITS": "5"}], ids=str)
@pytest.mark.parametrize("requests,heads,group,B,d,dtype", [
    (4, 8, 4, 4096, 128, roco.ROCO_BF16), (32, 8, 4, 2048, 128, roco.ROCO_BF16), (1, 8, 8, 20000, 64, roco.ROCO_BF16), (5, 5, 3, 1501, 128, roco.ROCO_F32),
    (2, 4, 2, 256, 128, roco.ROCO_BF16), (1, 1, 1, 7, 64, roco.ROCO_F32), (40, 1, 64, 300, 64, roco.ROCO_F32)])
def test_a_workspace_for_more_tokens_holds_fewer(env, requests, heads, group, B, d, dtype, monkeypatch):
    """One allocation, for the largest step, serves every smaller one of the same caches: what a call asks for does not fall as its tokens rise."""
    for name, value in env.items():
        monkeypatch.setenv(name, value)
    p = roco.RocoParams(requests * heads, d, B, 1, dtype)
    sizes = [roco.chunk_workspace_bytes(p, heads, group, t) for t in [*range(1, 1200), *range(1200, 20000, 171), 1 << 17, 1 << 20]]
    assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_small_tiles_are_not_asked_for_beyond_a_launch(monkeypatch):
    """ROCO_CHUNK_ROWS=32 where as many tiles would be more workgroups than a launch has: the call takes the tiles that it takes by itself, to be seen by its workspace."""
    p = roco.RocoParams(1, 128, 256, 1, roco.ROCO_BF16)
    monkeypatch.setenv("ROCO_CHUNK_ROW_SPLITS", "1")
    tokens = [1 << 22, (1 << 23) - 1, 1 << 23, 1 << 24]  # times 64 / 32
    by_itself = [roco.chunk_workspace_bytes(p, 1, 64, t) for t in tokens]
    monkeypatch.setenv("ROCO_CHUNK_ROWS", "32")
    asked = [roco.chunk_workspace_bytes(p, 1, 64, t) for t in tokens]
    assert asked[0] < by_itself[0] and asked[1:] == by_itself[1:]


def _verify(dtype=roco.ROCO_F32, requests=3, nodes=8, vocab=1000, p=OK, p_strides=(8000, 1000), q=OK, q_strides=(8000, 1000), ptrs=None, optional=(OK, OK), max_path=8,
            workspace=OK, ws=None):
    t = [OK] * 6 if ptrs is None else ptrs
    need = roco.verify_workspace_bytes(3, 8, 1000) if ws is None else ws
    return roco.load_library().roco_tree_verify(dtype, requests, nodes, vocab, p, *p_strides, q, *q_strides, t[0], *optional, t[1], t[2], 0, max_path, *t[3:], workspace,
                                                need, None)


def test_verification_is_checked():
    need = roco.verify_workspace_bytes(3, 8, 1000)
    assert need > 0 and _verify(ws=0) == _verify(ws=need - 1) == EWORKSPACE
    for kw in (dict(requests=0), dict(nodes=0), dict(vocab=0), dict(max_path=0), dict(max_path=9), dict(p=None), dict(p=OK + 2), dict(q=OK + 2), dict(p_strides=(8000, 999)),
               dict(p_strides=(-8000, 1000)), dict(q_strides=(8000, 999)), dict(q_strides=(8000, -1000)), dict(workspace=None), dict(workspace=OK + 8)):
        assert _verify(**kw) == EINVAL, kw
    for kw in (dict(dtype=2), dict(requests=65536), dict(nodes=65), dict(vocab=(1 << 22) + 1, p_strides=(0, 1 << 23), q_strides=(0, 1 << 23))):
        assert _verify(**kw, ws=1 << 50) == EUNSUPPORTED, kw
    assert _verify(q=None, q_strides=(0, 0), ws=0) == EWORKSPACE and _verify(optional=(None, None), ws=0) == EWORKSPACE and _verify(dtype=roco.ROCO_BF16, p=OK + 2, ws=0) == EWORKSPACE
    assert _verify(optional=(OK + 2, OK)) == _verify(optional=(OK, OK + 2)) == EINVAL
    for i in range(6):
        assert _verify(ptrs=[OK + 4 if j == i else OK for j in range(6)], ws=0) == EWORKSPACE
        for bad in (None, OK + 2):
            assert _verify(ptrs=[bad if j == i else OK for j in range(6)]) == EINVAL
    assert roco.verify_workspace_bytes(0, 8, 1000) == roco.verify_workspace_bytes(3, 65, 1000) == roco.verify_workspace_bytes(3, 8, 0) == 0


def _rows(tokens=10, heads=4, group=2, d=128, dtype=torch.bfloat16):
    qkv = torch.zeros((tokens, heads * group + 2 * heads, d), dtype=dtype)
    return qkv[:, :heads * group], qkv[:, heads * group:-heads], qkv[:, -heads:]


def _through_the_binding():
    """Arguments reach the library in their places; what is no such argument is refused before it."""
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    f32 = lambda *s: torch.zeros(s)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, k, v = _rows()
    cache, pos, used = (bf(8, 256, 128), bf(8, 256, 128)), i32(8, 256), i32(8)
    attend = dict(pages=None, q=q, k_new=k, v_new=v, token_start=i32(3), qpos0=i32(2), K_cache=cache[0], V_cache=cache[1], pos=pos, n_used=used, out=bf(10, 8, 128),
                  lse=f32(10, 8), workspace=i32(4), workspace_bytes=0, stream=0)
    commit = {**attend, "stats": f32(8, 3, 256), "evicted_slot": i32(10, 4), "evicted_pos": None}
    del commit["out"]

    def code(call, kw, **more):
        with pytest.raises(roco.RocoError) as e:
            call(P, 4, 2, **{**kw, **more})
        return e.value.code

    def wrong(call, kw, error=ValueError, **more):
        with pytest.raises(error):
            call(P, 4, 2, **{**kw, **more})

    for call, kw in ((roco.roco_chunk_attend, attend), (roco.roco_chunk_commit, commit)):
        assert code(call, kw) == code(call, kw, q=q.view(10, 8, 128).unflatten(1, (4, 2))) == code(call, kw, pages=_pages()) == EWORKSPACE
        assert code(call, kw, pages=_pages(page=24)) == EINVAL
        assert code(call, kw, q=bf(10, 8, 128), k_new=bf(10, 4, 128), v_new=bf(10, 4, 128)) == EWORKSPACE
        wrong(call, kw, q=bf(10, 7, 128))
        wrong(call, kw, q=bf(9, 8, 128))
        wrong(call, kw, q=bf(10, 128, 8).transpose(1, 2))
        wrong(call, kw, k_new=bf(10, 4, 128))  # V lies otherwise
        wrong(call, kw, q=q.float())
        wrong(call, kw, q=q.float(), k_new=k.float(), v_new=v.float())  # not the parameters' type
        wrong(call, kw, token_start=i32(2))
        wrong(call, kw, qpos0=i32(8))
        wrong(call, kw, token_start=torch.zeros(3, dtype=torch.int64))
        wrong(call, kw, qpos0=f32(2))
        wrong(call, kw, pos=pos.long())
        wrong(call, kw, n_used=used.float())
        wrong(call, kw, lse=f32(10, 7))
        wrong(call, kw, lse=f32(10, 8).double())
        wrong(call, kw, K_cache=bf(256, 8, 128).transpose(0, 1))
        wrong(call, kw, TypeError, pages=7)
        none = {"q": q[:0], "k_new": k[:0], "v_new": v[:0], "lse": f32(0, 8)}
        none.update({"out": bf(0, 8, 128)} if "out" in kw else {"evicted_slot": None})
        call(P, 4, 2, **{**kw, **none})  # no tokens: nothing is done
    wrong(roco.roco_chunk_attend, attend, out=bf(10, 8, 64))
    wrong(roco.roco_chunk_attend, attend, out=f32(10, 8, 128))
    assert code(roco.roco_chunk_attend, attend, lse=None) == EWORKSPACE
    wrong(roco.roco_chunk_commit, commit, stats=f32(8, 3, 256).double())
    wrong(roco.roco_chunk_commit, commit, evicted_slot=i32(10, 3))
    wrong(roco.roco_chunk_commit, commit, evicted_pos=i32(10, 4).long())

    p = torch.zeros((3, 8, 1000))
    verify = dict(p=p, q=p.clone(), tokens=i32(3, 8), parent=None, n_nodes=None, accept=f32(3, 8), choose=f32(3), path=i32(3, 8), n_path=i32(3), next_token=i32(3),
                  workspace=i32(4), workspace_bytes=0, stream=0)

    def refused(**kw):
        with pytest.raises(roco.RocoError) as e:
            roco.roco_tree_verify(**{**verify, **kw})
        return e.value.code

    assert refused() == refused(q=None) == refused(parent=i32(3, 8), n_nodes=i32(3), distinct=True) == refused(path=i32(3, 5)) == EWORKSPACE
    assert refused(p=torch.zeros((3, 8, 1003))[..., :1000]) == refused(q=p[:1].expand(3, -1, -1)) == EWORKSPACE
    assert refused(path=i32(3, 9)) == refused(path=i32(3, 0)) == refused(p=p[:, :1].expand(-1, 8, -1)) == EINVAL
    assert refused(p=p.half(), q=p.half()) == EUNSUPPORTED
    for kw in (dict(q=p[:2]), dict(q=p.bfloat16()), dict(p=torch.zeros((3, 1000, 8)).transpose(1, 2)), dict(tokens=i32(3, 7)), dict(accept=f32(3, 8).double()),
               dict(choose=f32(4)), dict(parent=i32(24)), dict(n_nodes=i32(4)), dict(path=i32(2, 8)), dict(path=i32(24)), dict(n_path=i32(3).long()), dict(next_token=f32(3)),
               dict(tokens=i32(3, 8).long()), dict(p=p[0])):
        with pytest.raises(ValueError):
            roco.roco_tree_verify(**{**verify, **kw})


def test_through_the_extension():
    _through_the_binding()


def test_through_ctypes_alone(monkeypatch):
    monkeypatch.setattr(binding, "_NATIVE_NAME", "_not_built")
    monkeypatch.setattr(binding, "_native_lib", None)
    monkeypatch.setattr(binding, "_marshal", None, raising=False)
    _through_the_binding()
    assert isinstance(binding._marshal, binding._PlainCalls)
