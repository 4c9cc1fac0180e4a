"""Refusals of the drafted trees' and pages' entry points, all on the host (no GPU: nothing is launched), through the C ABI, the
extension module and ctypes alone."""
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


def _attend(params=P, heads=4, group=2, nodes=8, pages=None, ws=None, ptrs=None, optional=(OK, OK, OK)):
    p = [OK] * 10 if ptrs is None else ptrs
    need = roco.tree_workspace_bytes(params, 2, 8) if ws is None else ws
    parent, n_nodes, lse = optional
    return roco.load_library().roco_tree_attend(ctypes.byref(params), heads, group, nodes, None if pages is None else ctypes.byref(pages), p[0], p[1],
                                                p[2], parent, n_nodes, p[3], p[4], p[5], p[6], p[7], p[8], lse, p[9], need, None)


def _commit(params=P, heads=4, group=2, nodes=8, pages=None, max_path=4, ws=None, ptrs=None, optional=(OK, OK)):
    p = [OK] * 13 if ptrs is None else ptrs
    need = roco.tree_workspace_bytes(params, 2, 8) if ws is None else ws
    return roco.load_library().roco_tree_commit(ctypes.byref(params), heads, group, nodes, None if pages is None else ctypes.byref(pages), *p[:4],
                                                max_path, *p[4:12], *optional, p[12], need, None)


@pytest.mark.parametrize("call", [_attend, _commit])
def test_shapes_are_checked(call):
    assert call(ws=0) == EWORKSPACE  # everything else is in order
    need = roco.tree_workspace_bytes(P, 2, 8)
    assert need > 0 and call(ws=need - 1) == EWORKSPACE
    assert call(heads=0) == EINVAL and call(heads=3) == EINVAL and call(heads=-4) == EINVAL  # 8 units
    assert call(group=0) == EINVAL and call(nodes=0) == EINVAL
    assert call(group=65) == EUNSUPPORTED and call(nodes=65) == EUNSUPPORTED
    for kw, code in ((dict(units=0), EINVAL), (dict(scope=257), EINVAL), (dict(head_dim=96), EUNSUPPORTED), (dict(dtype=2), EUNSUPPORTED),
                     (dict(scale=float("nan")), EINVAL), (dict(recency_window=-1), EINVAL), (dict(units=65536), EUNSUPPORTED)):
        bad = roco.RocoParams(**{**dict(units=8, head_dim=128, budget=256, scope=16, dtype=roco.ROCO_BF16), **kw})
        assert call(bad, ws=1 << 40) == code
        assert roco.tree_workspace_bytes(bad, 2, 8) == 0
    assert call(roco.RocoParams(65532, 128, 1 << 17, 16, roco.ROCO_BF16), ws=1 << 50) == EUNSUPPORTED  # 2^33 rows without pages
    assert roco.tree_workspace_bytes(P, 0, 8) == roco.tree_workspace_bytes(P, 2, 65) == 0


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
    for i in range(10):
        words = i in (3, 6, 7)  # qpos0, pos, n_used
        assert _attend(ptrs=[OK + 4 if j == i else OK for j in range(10)], ws=0) == (EWORKSPACE if words else EINVAL)
        for bad in (None, OK + (2 if words else 8)):
            assert _attend(ptrs=[bad if j == i else OK for j in range(10)]) == EINVAL
    for i in range(13):
        words = i in (3, 4, 5, 6, 9, 10, 11)  # lse, path, n_path, qpos0, stats, pos, n_used
        assert _commit(ptrs=[OK + 4 if j == i else OK for j in range(13)], ws=0) == (EWORKSPACE if words else EINVAL)
        for bad in (None, OK + (2 if words else 8)):
            assert _commit(ptrs=[bad if j == i else OK for j in range(13)]) == EINVAL
    for i in range(3):
        assert _attend(optional=[None if j == i else OK for j in range(3)], ws=0) == EWORKSPACE
        assert _attend(optional=[OK + 2 if j == i else OK for j in range(3)]) == EINVAL
    for i in range(2):
        assert _commit(optional=[None if j == i else OK for j in range(2)], ws=0) == EWORKSPACE
        assert _commit(optional=[OK + 2 if j == i else OK for j in range(2)]) == EINVAL
    assert _commit(max_path=0) == EINVAL and _commit(max_path=9) == EINVAL  # 8 nodes
    assert roco.load_library().roco_tree_attend(None, 1, 1, 1, None, *[OK] * 13, 0, None) == EINVAL


def test_tables_and_stores_are_checked():
    lib = roco.load_library()

    def tables(requests=4, page=64, max_pages=4, ptrs=(OK,) * 7, n_free=9, rows=10):
        return lib.roco_page_tables(requests, page, max_pages, ptrs[0], ptrs[1], ptrs[2], n_free, ptrs[3], ptrs[4], ptrs[5], ptrs[6], rows, 0, None)

    for i in range(7):  # (all but `held` are needed)
        odd = OK + (8 if i == 6 else 2)  # (the map is written 16 bytes at a time)
        assert tables(ptrs=[odd if j == i else OK for j in range(7)]) == EINVAL
        if i > 0:
            assert tables(ptrs=[None if j == i else OK for j in range(7)]) == EINVAL
    for kw in (dict(requests=0), dict(page=24), dict(page=0), dict(max_pages=0), dict(n_free=-1), dict(rows=0)):
        assert tables(**kw) == EINVAL
    assert tables(requests=65536) == EUNSUPPORTED and tables(max_pages=1 << 25) == EUNSUPPORTED

    def store(dtype=roco.ROCO_BF16, d=128, heads=2, groups=1, rows=5, strides=(0, 256, 128), ptrs=(OK,) * 5, n_pages=4, page=16):
        return lib.roco_page_store(dtype, d, heads, groups, rows, ptrs[0], ptrs[1], *strides, *ptrs[2:], n_pages, page, None)

    for i in range(5):
        for bad in (None, OK + (2 if i == 2 else 8)):
            assert store(ptrs=[bad if j == i else OK for j in range(5)]) == EINVAL
    for kw in (dict(heads=0), dict(groups=0), dict(rows=0), dict(n_pages=0), dict(page=17), dict(strides=(0, 256, -128)),
               dict(strides=(0, 252, 128)), dict(strides=(4, 256, 128))):
        assert store(**kw) == EINVAL
    for kw in (dict(dtype=3), dict(d=96), dict(n_pages=1 << 26)):
        assert store(**kw) == EUNSUPPORTED


def _through_the_binding():
    """Arguments reach the library in their places; what is no such argument is refused before it."""
    ten = [OK] * 13
    with pytest.raises(roco.RocoError) as e:
        roco.roco_tree_attend(P, 4, 2, 8, _pages(), *ten, workspace_bytes=0, stream=0)
    assert e.value.code == EWORKSPACE
    with pytest.raises(roco.RocoError) as e:
        roco.roco_tree_attend(P, 3, 2, 8, None, *ten, workspace_bytes=0, stream=0)
    assert e.value.code == EINVAL
    with pytest.raises(TypeError, match="RocoPages"):
        roco.roco_tree_attend(P, 4, 2, 8, 7, *ten, workspace_bytes=0, stream=0)
    with pytest.raises(ValueError, match="contiguous"):
        roco.roco_tree_attend(P, 4, 2, 8, None, torch.empty(8, 8).t(), *ten[1:], workspace_bytes=0, stream=0)
    for max_path, code in ((4, EWORKSPACE), (9, EINVAL)):
        with pytest.raises(roco.RocoError) as e:
            roco.roco_tree_commit(P, 4, 2, 8, _pages(), *[OK] * 4, max_path, *[OK] * 11, workspace_bytes=0, stream=0)
        assert e.value.code == code
    with pytest.raises(TypeError, match="RocoPages"):
        roco.roco_tree_commit(P, 4, 2, 8, P, *[OK] * 4, 4, *[OK] * 11, workspace_bytes=0, stream=0)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(roco.RocoError) as e:
        roco.roco_page_tables(i32(3), i32(3), 24, i32(4), i32(3, 2), i32(4), i32(4), i32(9), stream=0)
    assert e.value.code == EINVAL
    for bad in ((i32(2), i32(3), i32(4), i32(4), i32(9)), (i32(3), i32(2), i32(4), i32(4), i32(9)), (i32(3), i32(3), i32(3), i32(4), i32(9)),
                (i32(3), i32(3), i32(4), i32(3), i32(9)), (i32(3), i32(3), i32(4), i32(4), i32(2, 9))):
        with pytest.raises(ValueError):
            roco.roco_page_tables(bad[0], bad[1], 16, i32(4), i32(3, 2), *bad[2:], stream=0)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(roco.RocoError) as e:
        roco.roco_page_store(bf(5, 2, 128), bf(5, 2, 128), i32(5), bf(3, 2, 24, 128), bf(3, 2, 24, 128), stream=0)
    assert e.value.code == EINVAL
    with pytest.raises(roco.RocoError) as e:
        roco.roco_page_store(bf(5, 2, 132)[..., :128], bf(5, 2, 132)[..., :128], i32(5), bf(3, 2, 16, 128), bf(3, 2, 16, 128), stream=0)
    assert e.value.code == EINVAL  # rows at strides of 264 bytes
    pool = bf(3, 2, 16, 128)
    for k, v, m, pools in ((bf(5, 3, 128), bf(5, 3, 128), i32(5), (pool, pool)), (bf(5, 2, 128), bf(4, 2, 128), i32(5), (pool, pool)),
                           (bf(5, 2, 128), bf(5, 2, 128), i32(4), (pool, pool)), (bf(2, 2, 5, 128), bf(2, 2, 5, 128), i32(5), (pool, pool)),
                           (bf(5, 2, 128), bf(2, 5, 128).transpose(0, 1), i32(5), (pool, pool)), (bf(128, 2, 5).permute(2, 1, 0), bf(128, 2, 5).permute(2, 1, 0), i32(5), (pool, pool)),
                           (bf(5, 2, 128).float(), bf(5, 2, 128), i32(5), (pool, pool)), (bf(5, 2, 128), bf(5, 2, 128), i32(5), (pool, bf(4, 2, 16, 128)))):
        with pytest.raises(ValueError):
            roco.roco_page_store(k, v, m, *pools, stream=0)
    half = torch.zeros((3, 2, 16, 128), dtype=torch.float16)
    with pytest.raises(roco.RocoError) as e:
        roco.roco_page_store(half[:, :, 0], half[:, :, 0], i32(3), half, half, stream=0)
    assert e.value.code == EUNSUPPORTED


def test_through_the_extension():
    _through_the_binding()


def test_through_ctypes_alone(monkeypatch):
    monkeypatch.setattr(binding, "_NATIVE_NAME", "_not_built")
    monkeypatch.setattr(binding, "_native_lib", None)
    monkeypatch.setattr(binding, "_marshal", None, raising=False)
    _through_the_binding()
    assert isinstance(binding._marshal, binding._PlainCalls)


def test_the_structure_matches_the_header():
    assert ctypes.sizeof(roco.RocoPages) == 32
    assert [f[0] for f in roco.RocoPages._fields_] == ["table", "budget", "max_pages", "page", "n_pages"]
    table = torch.zeros((6, 5), dtype=torch.int32)
    pages = roco.RocoPages(table, 9, 64)
    assert (pages.table, pages.budget, pages.max_pages, pages.page, pages.n_pages) == (table.data_ptr(), None, 5, 64, 9)


def _types_of_words():
    """Integers are int32, statistics and normalisers float32: a tensor of another type is refused before anything is read as what it is not."""
    t = lambda dtype: torch.zeros((8, 8), dtype=dtype)  # noqa: E731

    def refused(call, args, at, good, bads, **kw):
        args = list(args)
        for bad in bads:
            args[at] = t(bad)
            with pytest.raises(ValueError, match=str(good).split(".")[1]):
                call(*args, **kw)
            args[at] = torch.nn.Parameter(t(bad), requires_grad=False)
            with pytest.raises(ValueError, match=str(good).split(".")[1]):
                call(*args, **kw)
        args[at] = t(good)
        with pytest.raises(roco.RocoError):  # (the sizes are wrong)
            call(*args, **kw)

    ints, floats = (torch.int64, torch.int16, torch.float32), (torch.float64, torch.bfloat16, torch.int32)
    attend = [P, 4, 2, 8, _pages(), *[OK] * 13]
    for at in (8, 9, 10, 13, 14):  # parent, n_nodes, qpos0, pos, n_used
        refused(roco.roco_tree_attend, attend, at, torch.int32, ints, workspace_bytes=0, stream=0)
    refused(roco.roco_tree_attend, attend, 16, torch.float32, floats, workspace_bytes=0, stream=0)
    commit = [P, 4, 2, 8, _pages(), *[OK] * 4, 4, *[OK] * 11]
    for at in (10, 11, 12, 16, 17, 18, 19):  # path, n_path, qpos0, pos, n_used, evicted_slot, evicted_pos
        refused(roco.roco_tree_commit, commit, at, torch.int32, ints, workspace_bytes=0, stream=0)
    for at in (8, 15):
        refused(roco.roco_tree_commit, commit, at, torch.float32, floats, workspace_bytes=0, stream=0)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    tables = [i32(3), i32(3), 24, i32(4), i32(3, 2), i32(4), i32(4), i32(9)]  # (24 is no page size)
    for at in (0, 1, 3, 4, 5, 6, 7):
        for bad in ints:
            with pytest.raises(ValueError, match="int32"):
                roco.roco_page_tables(*[x.to(bad) if i == at else x for i, x in enumerate(tables)], stream=0)
    rows, pool = torch.zeros((5, 2, 128)), torch.zeros((3, 2, 24, 128))
    for bad in ints:
        with pytest.raises(ValueError, match="int32"):
            roco.roco_page_store(rows, rows, i32(5).to(bad), pool, pool, stream=0)
        with pytest.raises(ValueError, match="int32"):
            roco.RocoPages(i32(6, 5).to(bad), 9, 64)
        with pytest.raises(ValueError, match="int32"):
            roco.RocoPages(i32(6, 5), 9, 64, i32(6).to(bad))


def test_types_of_words_through_the_extension():
    _types_of_words()


def test_types_of_words_through_ctypes_alone(monkeypatch):
    monkeypatch.setattr(binding, "_NATIVE_NAME", "_not_built")
    monkeypatch.setattr(binding, "_native_lib", None)
    monkeypatch.setattr(binding, "_marshal", None, raising=False)
    _types_of_words()
    assert isinstance(binding._marshal, binding._PlainCalls)


def test_a_map_of_no_entries():
    lib = roco.load_library()
    # (of 65536 requests: refused, but only behind the checks of the arguments)
    tables = lambda rows, slot_map: lib.roco_page_tables(65536, 64, 4, OK, OK, OK, 9, OK, OK, OK, slot_map, rows, 0, None)  # noqa: E731
    assert tables(0, None) == EUNSUPPORTED and tables(1, OK) == EUNSUPPORTED
    assert tables(0, OK) == EINVAL and tables(1, None) == EINVAL and tables(-1, None) == EINVAL
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for slot_map in (None, i32(0), i32(3, 0)):
        with pytest.raises(roco.RocoError) as e:
            roco.roco_page_tables(i32(3), i32(3), 24, None, i32(3, 2), i32(4), i32(4), slot_map, stream=0)
        assert e.value.code == EINVAL  # 24 is no page size
    with pytest.raises(ValueError, match="padded"):
        roco.roco_page_tables(i32(3), i32(3), 16, None, i32(3, 2), i32(4), i32(4), i32(2, 0), stream=0)
    pool, none = torch.zeros((3, 2, 16, 128)), torch.zeros((0, 2, 128))
    roco.roco_page_store(none, none, i32(0), pool, pool, stream=0)
    for bad in (torch.zeros((0, 3, 128)), torch.zeros((0, 2, 64)), none.bfloat16()):
        with pytest.raises(ValueError):
            roco.roco_page_store(bad, bad, i32(0), pool, pool, stream=0)
    with pytest.raises(ValueError):
        roco.roco_page_store(none, none, i32(1), pool, pool, stream=0)


def test_a_store_of_more_than_a_launch_takes():
    store = lambda groups, rows, heads=8: roco.load_library().roco_page_store(  # noqa: E731
        roco.ROCO_F32, 128, heads, groups, rows, OK, OK, 0, 0, 0, OK, OK, OK, 4, 16, None)
    assert store((1 << 31) - 1, (1 << 31) - 1) == EUNSUPPORTED and store(1 << 20, 1 << 24) == EUNSUPPORTED  # (2^49 lanes, then 2^52)


@pytest.mark.parametrize("call", [_attend, _commit])
def test_large_calls_on_pages_have_a_workspace(call):
    """2^32 slots and more in all: too many for dense caches, not for pages."""
    large = roco.RocoParams(16384, 128, 1 << 18, 16, roco.ROCO_BF16)
    need = roco.tree_workspace_bytes(large, 2, 8)
    assert need > 8 << 32  # a sum of either kind per slot
    pages = _pages(max_pages=1 << 12)
    assert call(large, pages=pages, ws=need - 1) == EWORKSPACE
    assert call(large, ws=need) == EUNSUPPORTED  # without pages
    # ... as far as a launch goes: the query and the calls agree
    for units, budget in ((65532, 1 << 18), (65532, 1 << 20), (16384, 1 << 20), (1024, 1 << 24), (1020, 1 << 24)):
        p = roco.RocoParams(units, 128, budget, 16, roco.ROCO_BF16)
        fits = units * budget < 1 << 34
        need = roco.tree_workspace_bytes(p, 2, 8)
        assert (need > 0) == fits
        assert call(p, pages=_pages(max_pages=1 << 18), ws=max(need, 1) - 1) == (EWORKSPACE if fits else EUNSUPPORTED)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("units,budget,nodes,group", [(65535, 4096, 64, 64), (65535, 65000, 64, 1), (4100, 1 << 20, 64, 64), (4097, 9000, 64, 63), (64, 4096, 64, 64)])
def test_asked_splits_are_as_many_as_launches_take(monkeypatch, dtype, units, budget, nodes, group):
    """The workspace of the shares tells how many there are: 64 asked for."""
    p = roco.RocoParams(units, 64, budget, 16, dtype)
    commit = roco.tree_workspace_bytes(p, 1, 1)
    monkeypatch.setenv("ROCO_TREE_SPLITS", "64")
    rows = nodes * group
    splits = max(0, roco.tree_workspace_bytes(p, group, nodes) - commit) // (units * rows * 4 * 66)
    tile = 64 if dtype == 0 else 192
    assert -(-units * max(splits, 1) // 8) * 8 * -(-rows // tile) < 1 << 24
    assert splits <= 8 or units * rows < 1 << 24
