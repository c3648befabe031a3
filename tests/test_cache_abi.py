"""The paged cache's calls without a GPU: what they refuse, on the host and
before any launch (null device pointers are never followed), workspace sizes,
and the binding's and PagedCache's own checks."""

import ctypes
import os

import pytest
import torch

from cache_model import Model
from paper_2609_27373_amd import wise
from paper_2609_27373_amd.cache import PagedCache

OK, NULL, SHAPE, UNSUPPORTED, RANGE, WORKSPACE = range(6)
F = ctypes.c_void_p(4096)           # aligned, never followed
ODD = ctypes.c_void_p(4096 + 2)
HALF = ctypes.c_void_p(4096 + 8)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(wise.LIB_PATH):
        from paper_2609_27373_amd import build
        build.build()
    return wise.load()


def C(**kw):
    return wise.make_cache(**dict(dict(pages=10, page=32, kv_heads=2, head_dim=64, planes=2, seqs=4, max_pages=8), **kw))


def call(fn, c, **kw):
    """One C call with every pointer valid but those named."""
    i32 = ctypes.c_int32
    order = {
        "fork": [("n", 1), ("src", F), ("dst", F), ("tables", F), ("lens", F), ("refs", F), ("done", None)],
        "trim": [("n", 1), ("ids", F), ("new_lens", None), ("tables", F), ("lens", F), ("refs", F)],
        "reserve": [("n", 1), ("ids", F), ("counts", F), ("tables", F), ("lens", F), ("refs", F), ("granted", F), ("pool", F), ("ws", F),
                    ("wsb", 1 << 40)],
        "append": [("n", 1), ("tokens", 1), ("ids", F), ("counts", F), ("k", F), ("v", F), ("tables", F), ("lens", F), ("kp", F), ("vp", F)],
        "compact": [("tables", F), ("refs", F), ("pool", F), ("live", None), ("ws", F), ("wsb", 1 << 40)],
        "shared": [("batch", 1), ("least", 1), ("ids", None), ("tables", F), ("lens", F), ("out", F)],
        "attn": [("a", wise.make_queries(2, 4)), ("q", F), ("kp", F), ("vp", F), ("tables", F), ("lens", F), ("ids", None),
                 ("shared", None), ("o", F), ("lse", None), ("ws", F), ("wsb", 1 << 40)]}[fn]
    args = [kw.pop(name, default) for name, default in order]
    assert not kw
    args = [ctypes.byref(x) if isinstance(x, wise.wise_queries) else ctypes.c_size_t(x) if name == "wsb" else i32(x) if isinstance(x, int)
            else x for x, (name, _) in zip(args, order)]
    entry = "wise_prefix_attn" if fn == "attn" else "wise_cache_" + fn
    return getattr(wise.load(), entry)(ctypes.byref(c) if c is not None else None, *args, None)


CALLS = ("fork", "trim", "reserve", "append", "compact", "shared", "attn")


@pytest.mark.parametrize("fn", CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(pages=0), SHAPE), (dict(page=-16), SHAPE), (dict(kv_heads=0), SHAPE), (dict(planes=0), SHAPE), (dict(seqs=-1), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=256), UNSUPPORTED),
    (dict(head_dim=80), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(max_pages=1 << 26), SHAPE), (dict(max_pages=(1 << 25) + 1), SHAPE), (dict(planes=65536, kv_heads=17), SHAPE), (dict(pages=(1 << 27) + 1), SHAPE),
    (dict(kv_heads=1 << 20), SHAPE)])
def test_geometry(fn, kw, status):
    assert call(fn, C(**kw)) == status
    assert call(fn, None) == NULL
    assert wise.wise_cache_workspace_bytes(C(**kw)) == 0
    assert wise.wise_prefix_workspace_bytes(C(**kw), wise.make_queries(2, 4)) == 0


@pytest.mark.parametrize("fn,names", [
    ("fork", "src dst tables lens refs"), ("trim", "ids tables lens refs"),
    ("reserve", "ids counts tables lens refs granted pool ws"), ("append", "ids counts k v tables lens kp vp"),
    ("compact", "tables refs pool ws"), ("shared", "tables lens out"), ("attn", "q kp vp tables lens o ws")])
def test_pointers(fn, names):
    for name in names.split():
        assert call(fn, C(), **{name: None}) == NULL, name
        assert call(fn, C(), **{name: ODD}) == SHAPE, name
        if name in ("pool", "k", "v", "kp", "vp", "q", "o", "ws"):
            assert call(fn, C(), **{name: HALF}) == SHAPE, name
    for name in {"fork": ["done"], "trim": ["new_lens"], "compact": ["live"], "shared": ["ids"], "attn": ["ids", "shared", "lse"]}.get(fn, []):
        assert call(fn, C(), **{name: ODD}) == SHAPE, name


@pytest.mark.parametrize("fn", ["fork", "trim", "reserve", "append"])
def test_entries(fn):
    assert call(fn, C(), n=-1) == SHAPE
    assert call(fn, C(), n=1025) == UNSUPPORTED
    names = {"fork": ["src", "dst"], "trim": ["ids"], "reserve": ["ids", "counts", "granted"], "append": ["ids", "k", "v"]}[fn]
    assert call(fn, C(), n=0, **{x: None for x in names}) == OK      # nothing to do, nothing launched


def test_sizes():
    assert call("append", C(), tokens=0) == SHAPE
    assert call("append", C(), n=1024, tokens=1 << 20) == SHAPE      # 2^31 rows
    assert call("append", C(), n=1024, tokens=1 << 17) == SHAPE      # 2^28: more threads than a launch may have
    assert call("shared", C(), batch=0) == SHAPE
    assert call("shared", C(), batch=5) == SHAPE                      # 4 table rows
    assert call("shared", C(), batch=1025, ids=F) == UNSUPPORTED
    for fn in ("reserve", "compact"):
        need = wise.wise_cache_workspace_bytes(C())
        assert need > 0 and call(fn, C(), wsb=need - 1) == WORKSPACE


@pytest.mark.parametrize("a,status", [
    (None, NULL), (wise.make_queries(0, 4), SHAPE), (wise.make_queries(2, 0), SHAPE), (wise.make_queries(2, 4, 0), SHAPE),
    (wise.make_queries(2, 3), SHAPE), (wise.make_queries(5, 4), SHAPE), (wise.make_queries(1025, 4), UNSUPPORTED),
    (wise.make_queries(2, 4, 65), UNSUPPORTED), (wise.make_queries(2, 2 * 129), UNSUPPORTED), (wise.make_queries(2, 2, 1 << 30), UNSUPPORTED), (wise.make_queries(1024, 1 << 16), UNSUPPORTED),
    (wise.make_queries(2, 4, 1, float("nan")), RANGE), (wise.make_queries(2, 4, 1, float("-inf")), RANGE)])
def test_queries(a, status):
    assert call("attn", C(), a=a) == status
    if a is not None and a.batch != 5:
        assert wise.wise_prefix_workspace_bytes(C(), a) == 0


def test_more_queries_than_indexes():
    c = C(kv_heads=1 << 15, head_dim=64, page=16, seqs=1024)
    assert call("attn", c, a=wise.make_queries(1024, 1 << 15)) == SHAPE          # 2^31 elements of q
    assert wise.wise_prefix_workspace_bytes(c, wise.make_queries(1024, 1 << 15)) == 0
    assert wise.wise_prefix_workspace_bytes(c, wise.make_queries(1023, 1 << 15)) > 0
    assert wise.wise_cache_workspace_bytes(C(max_pages=1 << 25)) > 0


def test_largest_batches_have_a_workspace():
    c = PagedCache(1, 1, 16, 1 << 15, 64, 1024, 1, device="meta")
    assert wise.wise_prefix_workspace_bytes(c.shape, wise.make_queries(1024, 1 << 15)) == 0     # 2^31 elements of q
    for b in (600, 1023, 700, 600):
        assert c._attend_workspace(b, 1 << 15, 1)[1] >= wise.wise_prefix_workspace_bytes(c.shape, wise.make_queries(b, 1 << 15)) > 0
    assert len(c._attend) == 3                                          # kept: a captured graph goes on using its own


def test_attention_workspace():
    a = wise.make_queries(2, 4)
    need = wise.wise_prefix_workspace_bytes(C(), a)
    assert need > 0 and call("attn", C(), a=a, wsb=need - 1) == WORKSPACE
    sizes = [wise.wise_prefix_workspace_bytes(C(seqs=1024), wise.make_queries(b, 4, t)) for t in (1, 7, 64) for b in (1, 2, 3, 17, 1024)]
    assert all(x <= y for x, y in zip(sizes, sizes[1:5])) and all(s > 0 for s in sizes)


def test_binding_refuses_host_tensors():
    c = C()
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        wise.wise_cache_fork(c, t, t, t, t, t)
    with pytest.raises(ValueError):
        wise.wise_cache_shared(c, 4, 1, None, t, t, t)


def test_paged_cache_checks():
    make = lambda **kw: PagedCache(**dict(dict(layers=2, pages=6, page=16, kv_heads=2, head_dim=64, seqs=3, max_pages=4, device="cpu"), **kw))  # noqa: E731
    c = make()
    assert c.pool.shape == (4, 6, 2, 16, 64) and c.tables.unique().tolist() == [-1] and c.lens.sum() == c.refs.sum() == 0
    for bad in (dict(page=24), dict(head_dim=100), dict(layers=0), dict(seqs=0)):
        with pytest.raises(ValueError):
            make(**bad)
    with pytest.raises(ValueError):
        make(pool=torch.zeros(4, 6, 2, 16, 64))
    with pytest.raises(ValueError):
        make(lens=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        c.layer(2)
    ids, one = torch.zeros(1, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    bf = dict(dtype=torch.bfloat16)
    for k, v in ((torch.zeros(1, 2, 3, 32, **bf),) * 2, (torch.zeros(2, 2, 3, 64, **bf),) * 2,
                 (torch.zeros(1, 2, 3, 64, **bf), torch.zeros(1, 2, 4, 64, **bf))):
        with pytest.raises(ValueError):
            c.append(0, k, v, ids, one)
    with pytest.raises(ValueError):
        c.attend(0, torch.zeros(1, 4, 1, 64, **bf), torch.zeros(1, 4, 2, 64, **bf))


def test_model_by_hand():
    """The plain model on a case worked out by hand."""
    m = Model(2, 6, 4, 1, 1, 4, 3, list(range(48)))
    assert m.reserve([1, 0, 1], [5, 4, 1]) == [5, 4, 0]
    assert m.tables[1] == [0, 1, -1] and m.tables[0] == [2, -1, -1] and m.refs == [1, 1, 1, 0, 0, 0]
    assert m.fork([1, 1], [2, 2]) == [1, 0] and m.refs == [2, 2, 1, 0, 0, 0]
    assert m.shared([1, 2, 0]) == [0, 1, 0]
    assert m.reserve([2, 1], [1, 1]) == [1, 1]       # both copy page 1, which nobody names then
    assert m.tables[2] == [0, 3, -1] and m.tables[1] == [0, 4, -1] and m.refs == [2, 0, 1, 1, 1, 0]
    assert m.pool[:, 3, 0, 0].tolist() == m.pool[:, 1, 0, 0].tolist() == [[4], [28]] and m.pool[0, 3, 0, 1, 0] == 13
    assert m.counts_hold() and m.compact() == 4
    assert m.tables[1] == [0, 1, -1] and m.refs == [2, 1, 1, 1, 0, 0] and m.counts_hold()
    m.trim([2, 0], [4, 0])
    assert m.tables[2] == [0, -1, -1] and m.lens == [0, 6, 4, 0] and m.counts_hold()


def test_append_rows_that_one_launch_holds():
    """2^28 - 1 and 2^28 - 15 rows round up to 2^24 groups of 256 threads at head_dim 128: 2^32, more than a launch may have."""
    for d in (64, 96, 128):
        assert 381 * 43 * 16385 == (1 << 28) - 1
        assert call("append", C(kv_heads=16385, page=16, head_dim=d), n=381, tokens=43) == SHAPE
        assert call("append", C(kv_heads=1, head_dim=d), n=1, tokens=(1 << 28) - 15) == SHAPE
        # The largest that is accepted, by both kernels: rows a group when tokens are few; tiles of 32 or 64 tokens.
        rows = (1 << 28) - 16
        few = -(-rows // (256 // (d // 8))) * 256
        many = max(-(-rows // t) * -(-t // (64 if d == 96 else 32)) * 256 for t in range(64, 4096))
        assert few < 1 << 32 and many < 1 << 32
