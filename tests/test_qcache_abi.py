"""The cache in 8 or 4 bits without a GPU: what its calls refuse before any launch (null
device pointers are never followed), sizes, QuantCache's own checks, and the plain model of
the tests by hand."""

import ctypes
import os

import numpy as np
import pytest
import torch

from kept_model import attend, pack, page_bytes, places, quantise, read, unpack, values
from paper_2609_27373_amd import wise
from paper_2609_27373_amd.cache import PagedCache, QuantCache

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


def call(fn, c, bits=4, **kw):
    """One C call with every pointer valid but those named."""
    i32 = ctypes.c_int32
    order = {
        "reserve": [("n", 1), ("ids", F), ("counts", F), ("tables", F), ("lens", F), ("refs", F), ("granted", F), ("pool", F), ("ws", F),
                    ("wsb", 1 << 40)],
        "append": [("n", 1), ("tokens", 1), ("ids", F), ("counts", F), ("k", F), ("v", F), ("tables", F), ("lens", F), ("kp", F), ("vp", F)],
        "read": [("n", 1), ("tokens", 1), ("ids", F), ("counts", F), ("starts", None), ("kp", F), ("vp", F), ("tables", F), ("lens", F), ("k", F),
                 ("v", F)],
        "compact": [("tables", F), ("refs", F), ("pool", F), ("live", None), ("ws", F), ("wsb", 1 << 40)],
        "attn": [("a", wise.make_queries(2, 4)), ("q", F), ("kp", F), ("vp", F), ("tables", F), ("lens", F), ("ids", None),
                 ("shared", None), ("o", F), ("lse", None), ("ws", F), ("wsb", 1 << 40)]}[fn]
    args = [kw.pop(name, default) for name, default in order]
    assert not kw
    args = [ctypes.byref(x) if isinstance(x, wise.wise_queries) else ctypes.c_size_t(x) if name == "wsb" else i32(x) if isinstance(x, int)
            else x for x, (name, _) in zip(args, order)]
    return getattr(wise.load(), "wise_qcache_" + fn)(ctypes.byref(c) if c is not None else None, i32(bits), *args, None)


CALLS = ("reserve", "append", "read", "compact", "attn")


@pytest.mark.parametrize("fn", CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(pages=0), SHAPE), (dict(page=-16), SHAPE), (dict(kv_heads=0), SHAPE), (dict(planes=0), SHAPE), (dict(seqs=-1), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(page=8), UNSUPPORTED), (dict(page=256), UNSUPPORTED), (dict(head_dim=80), UNSUPPORTED),
    (dict(max_pages=1 << 26), SHAPE), (dict(planes=65536, kv_heads=17), SHAPE), (dict(pages=(1 << 27) + 1), SHAPE), (dict(kv_heads=1 << 20), SHAPE)])
def test_geometry(fn, kw, status):
    assert call(fn, C(**kw)) == status
    assert call(fn, None) == NULL
    assert wise.wise_qcache_workspace_bytes(C(**kw), 4, wise.make_queries(2, 4)) == 0
    assert wise.wise_qcache_page_bytes(C(**kw), 4) == 0


@pytest.mark.parametrize("bits", [-4, 0, 1, 2, 3, 5, 6, 7, 9, 16, 32])
def test_widths(bits):
    for fn in CALLS:
        assert call(fn, C(), bits) == UNSUPPORTED
    assert wise.wise_qcache_page_bytes(C(), bits) == wise.wise_qcache_workspace_bytes(C(), bits, wise.make_queries(2, 4)) == 0
    with pytest.raises(ValueError):
        QuantCache(1, 4, 16, 2, 64, 3, 4, bits=bits, device="cpu")


@pytest.mark.parametrize("fn,names", [
    ("reserve", "ids counts tables lens refs granted pool ws"), ("append", "ids counts k v tables lens kp vp"),
    ("read", "ids counts k v tables lens kp vp"), ("compact", "tables refs pool ws"), ("attn", "q kp vp tables lens o ws")])
def test_pointers(fn, names):
    for name in names.split():
        assert call(fn, C(), **{name: None}) == NULL, name
        assert call(fn, C(), **{name: ODD}) == SHAPE, name
        if name in ("pool", "k", "v", "kp", "vp", "q", "o", "ws"):
            assert call(fn, C(), **{name: HALF}) == SHAPE, name
    for name in {"read": ["starts"], "compact": ["live"], "attn": ["ids", "shared", "lse"]}.get(fn, []):
        assert call(fn, C(), **{name: ODD}) == SHAPE, name


@pytest.mark.parametrize("fn", ["reserve", "append", "read"])
def test_entries(fn):
    assert call(fn, C(), n=-1) == SHAPE
    assert call(fn, C(), n=1025) == UNSUPPORTED
    assert call(fn, C(), n=0, ids=None) == OK                        # nothing to do, nothing launched
    if fn != "reserve":
        assert call(fn, C(), tokens=0) == SHAPE
        for d in (64, 96, 128):
            assert call(fn, C(kv_heads=16385, page=16, head_dim=d), n=381, tokens=43) == SHAPE       # 2^28 - 1 rows
            assert call(fn, C(kv_heads=1, head_dim=d), n=1, tokens=(1 << 28) - 15) == SHAPE


def test_rows_that_one_launch_holds():
    """16 threads for each four of positions that an entry's tokens reach into: fewer than 2^32 at the largest size accepted."""
    for tokens in (1, 2, 3, 4, 5, 43, 1 << 20, (1 << 28) - 16):
        rows = ((1 << 28) - 16) // tokens
        assert -(-rows * ((tokens + 6) // 4) // 16) * 256 < 1 << 32


@pytest.mark.parametrize("a,status", [
    (None, NULL), (wise.make_queries(0, 4), SHAPE), (wise.make_queries(2, 3), SHAPE), (wise.make_queries(5, 4), SHAPE),
    (wise.make_queries(1025, 4), UNSUPPORTED), (wise.make_queries(2, 4, 65), UNSUPPORTED), (wise.make_queries(2, 4, 1, float("nan")), RANGE)])
def test_queries(a, status):
    assert call("attn", C(), a=a) == status
    if a is not None and a.batch != 5:
        assert wise.wise_qcache_workspace_bytes(C(), 8, a) == 0


def test_workspaces():
    a = wise.make_queries(2, 4)
    for bits in (4, 8):
        need = wise.wise_qcache_workspace_bytes(C(), bits, a)
        assert need > 0 and call("attn", C(), bits, a=a, wsb=need - 1) == WORKSPACE
    for fn in ("reserve", "compact"):
        assert call(fn, C(), wsb=wise.wise_cache_workspace_bytes(C()) - 1) == WORKSPACE


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_page_bytes(d, bits):
    for page in (16, 32, 64, 128):
        n = wise.wise_qcache_page_bytes(C(page=page, head_dim=d), bits)
        assert n == page_bytes(page, d, bits) and n % 16 == 0


def test_quant_cache_checks():
    make = lambda **kw: QuantCache(**dict(dict(layers=2, pages=6, page=16, kv_heads=2, head_dim=96, seqs=3, max_pages=4, device="cpu"), **kw))  # noqa: E731
    c = make()
    assert isinstance(c, PagedCache) and c.bits == 4
    assert c.pool.shape == (4, 6, 2, 16 * 51) and c.pool.dtype == torch.uint8 and c.layer(1)[1].data_ptr() == c.pool[3].data_ptr()
    assert make(bits=8).pool.shape == (4, 6, 2, 16 * 99)
    pool = torch.ones((4, 6, 2, 16 * 51), dtype=torch.uint8)
    assert make(pool=pool).pool is pool
    for bad in (dict(page=24), dict(head_dim=100), dict(layers=0), dict(seqs=0), dict(pool=pool[:2]), dict(pool=pool.float()), dict(pool=pool, bits=8)):
        with pytest.raises(ValueError):
            make(**bad)
    ids, one, bf = torch.zeros(1, dtype=torch.int32), torch.ones(1, dtype=torch.int32), dict(dtype=torch.bfloat16)
    for k, v in ((torch.zeros(1, 2, 3, 64, **bf),) * 2, (torch.zeros(2, 2, 3, 96, **bf),) * 2, (torch.zeros(1, 2, 3, 96, **bf), torch.zeros(1, 2, 4, 96, **bf))):
        for fn in (c.append, c.read):
            with pytest.raises(ValueError):
                fn(0, k, v, ids, one)
    k = torch.zeros(1, 2, 3, 96, **bf)
    for layer in (-1, 2):
        with pytest.raises(ValueError):
            c.read(layer, k, k, ids, one)
    with pytest.raises(ValueError):
        c.read(0, k, k, ids, one)                                    # not on a GPU


def test_binding_refuses_host_tensors():
    c, t, b = C(), torch.zeros(4, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.bfloat16)
    p = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError):
        wise.wise_qcache_append(c, 4, 1, t, t, b, b, t, t, p, p)
    with pytest.raises(ValueError):
        wise.wise_qcache_read(c, 4, 1, t, t, None, p, p, t, t, b, b)


def test_model_by_hand():
    x = np.zeros((1, 64))
    x[0, :5] = [7, 2.5, -5, 0.25, -0.75]             # scale 1: 7 -> 6, 2.5 -> 2, -5 -> -4, 0.25 -> 0, -0.75 -> -1
    x[0, 32:34] = [7.25, 1]                          # scale 2: 3.625 -> 4, 0.5
    codes, scales = quantise(x, 4)
    assert scales.tolist() == [[127, 128]] and codes[0, :5].tolist() == [7, 4, 14, 0, 10] and codes[0, 32:34].tolist() == [6, 1]
    assert values(codes, scales, 4)[0, :5].tolist() == [6, 2, -4, 0, -1] and values(codes, scales, 4)[0, 32:34].tolist() == [8, 1]
    x[0, :5] = [464, 456, 17, -18, 2.0 ** -10]       # scale 1: 448, 448, 16 (tie), -18, 0 (tie)
    x[0, 32:34] = [np.inf, 1]
    codes, scales = quantise(x, 8)
    assert scales.tolist() == [[127, 255]] and values(codes, scales, 8)[0, :5].tolist() == [448, 448, 16, -18, 0]
    assert np.isnan(values(codes, scales, 8)[0, 32:]).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_layout_model(d, bits):
    """Every (token, dim) has a place of its own, and what is packed comes back."""
    for page in (16, 64):
        for plane in (0, 1):
            code, shift, scale = places(page, d, bits, plane)
            assert len(set(zip(code.ravel().tolist(), shift.ravel().tolist()))) == page * d
            assert sorted(set(code.ravel().tolist()) | set(scale.ravel().tolist())) == list(range(page_bytes(page, d, bits)))
            rng = np.random.default_rng(0)
            c, s = rng.integers(0, 1 << bits, (2, page, d)).astype(np.uint8), rng.integers(0, 256, (2, page, d // 32)).astype(np.uint8)
            back = unpack(pack(c, s, bits, plane), page, d, bits, plane)
            assert np.array_equal(back[0], c) and np.array_equal(back[1], s)
    # Values: token 5 of the first page lies in the second four, its dim 17 in sixteenth 17 // (d / 16).
    six = d // 16 * bits // 8
    at = 4 * (d * bits // 8) + 17 // (d // 16) * 4 * six + six + 17 % (d // 16) * bits // 8
    assert places(16, d, bits, 1)[0][5, 17] == at and places(16, d, bits, 0)[0][5, 17] == 5 * d * bits // 8 + 17 * bits // 8


def test_model_attention():
    """One head, three tokens, by hand; and a NaN scale."""
    q = np.zeros((1, 1, 1, 64))
    q[0, 0, 0, 0] = 8.0
    k, v = np.zeros((1, 1, 16, 64)), np.zeros((1, 1, 16, 64))
    k[0, 0, :3, 0] = [0, np.log(2), np.log(4)]
    v[0, 0, :3, 5] = [7, 0, 1]
    o, lse, bound, _ = attend(q, k, v, np.array([[0]]), [3], [0], 16, 1 / 8)
    assert abs(o[0, 0, 0, 5] - 11 / 7) < 1e-12 and abs(lse[0, 0, 0] - np.log(7)) < 1e-12 and bound[0, 0, 0, 5] > 2.0 ** -8
    raw = np.zeros(page_bytes(16, 64, 4), np.uint8)
    raw[16 * 32:] = 127
    raw[16 * 32 + 1] = 255
    assert np.isnan(read(raw, 16, 64, 4, 0)[0, 32:]).all() and (read(raw, 16, 64, 4, 0)[0, :32] == 0).all()
