"""The paged cache's bookkeeping and page moves on the GPU against the plain
model, entry for entry and bit for bit: forks, trims, room with copies of
shared pages, appends, compaction, shared leading pages; refused entries;
long random runs of all of them together."""

import random

import numpy as np
import pytest
import torch

from cache_model import Model
from paper_2609_27373_amd.cache import PagedCache
from parity_util import say

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bits(t):
    return t.view(torch.int16).cpu().numpy()


def pair(layers=1, pages=40, page=16, kv=2, d=64, seqs=8, max_pages=6, seed=0):
    g = torch.Generator().manual_seed(seed)
    pool = torch.randint(-2 ** 15, 2 ** 15, (2 * layers, pages, kv, page, d), generator=g, dtype=torch.int16)
    m = Model(2 * layers, pages, page, kv, d, seqs, max_pages, pool.numpy())
    c = PagedCache(layers, pages, page, kv, d, seqs, max_pages, pool=pool.cuda().view(torch.bfloat16))
    return c, m


def same(c, m, what=""):
    torch.cuda.synchronize()
    assert c.lens.cpu().tolist() == m.lens, what
    assert c.refs.cpu().tolist() == m.refs, what
    assert c.tables.cpu().tolist() == m.tables, what
    assert np.array_equal(bits(c.pool), m.pool), what


def kv_rows(c, n, tokens, seed):
    g = torch.Generator().manual_seed(seed)
    shape = (n, c.shape.kv_heads, tokens, c.shape.head_dim)
    return [torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, dtype=torch.int16) for _ in range(2)]


def grow(c, m, ids, counts, seed=1, tokens=None):
    """Room and contents for counts[i] tokens more, on both sides."""
    granted = c.reserve(ints(ids), ints(counts))
    want = m.reserve(ids, counts)
    assert granted.cpu().tolist() == want
    tokens = max([1] + counts) if tokens is None else tokens
    for layer in range(m.planes // 2):
        k, v = kv_rows(c, len(ids), tokens, seed + layer)
        c.append(layer, k.cuda().view(torch.bfloat16), v.cuda().view(torch.bfloat16), ints(ids), granted)
        m.append(layer, k.numpy(), v.numpy(), ids, want)
    return want


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_fork_and_copy_on_write(gpu_lib, page, d):
    """Samples of a prompt share its pages; the partly filled last one is copied to each when they grow."""
    c, m = pair(layers=2, page=page, d=d, kv=3)
    grow(c, m, [0], [2 * page + 5])
    assert c.fork(ints([0, 0, 0]), ints([3, 1, 7])).cpu().tolist() == m.fork([0, 0, 0], [3, 1, 7]) == [1, 1, 1]
    same(c, m, "fork")
    assert m.refs[:3] == [4, 4, 4]
    assert grow(c, m, [1, 3, 7], [1, page, 2], seed=5) == [1, page, 2]
    same(c, m, "copies")
    assert m.counts_hold() and m.refs[2] == 1
    grow(c, m, [0], [1], seed=9)                      # the last holder writes in place
    same(c, m, "in place")
    assert m.refs[2] == 1 and m.tables[0][2] == 2


def test_every_claimant_copies(gpu_lib):
    """All holders of a page grow in one call: each gets a copy, the page itself becomes free."""
    c, m = pair()
    grow(c, m, [0], [20])
    c.fork(ints([0, 0]), ints([1, 2]))
    m.fork([0, 0], [1, 2])
    grow(c, m, [2, 0, 1], [1, 1, 1], seed=3)
    same(c, m)
    assert m.refs[1] == 0 and m.counts_hold()


@pytest.mark.parametrize("case", ["twice", "not empty", "source is destination", "ids", "empty source"])
def test_refused_forks(gpu_lib, case):
    c, m = pair()
    grow(c, m, [0, 1], [17, 33])
    src, dst, done = {"twice": ([0, 1, 0], [4, 4, 5], [1, 0, 1]), "not empty": ([0, 0], [1, 3], [0, 1]),
                      "source is destination": ([0, 2, 1], [2, 3, 4], [1, 0, 1]),
                      "ids": ([0, 8, -1, 0, 1], [-1, 2, 3, 8, 2], [0, 0, 0, 0, 0]),
                      "empty source": ([5, 0], [6, 7], [1, 1])}[case]
    got = c.fork(ints(src), ints(dst)).cpu().tolist()
    assert got == m.fork(src, dst) == done
    same(c, m)


def test_trims(gpu_lib):
    c, m = pair()
    grow(c, m, [0, 1, 2, 3], [50, 33, 16, 1])
    for ids, new in (([0, 1], [33, 40]), ([0, 0, 1], [32, 0, -4]), ([2, 9, -1, 2], [15, 0, 0, 3]), ([3, 1, 0], None), ([0], None)):
        c.trim(ints(ids), None if new is None else ints(new))
        m.trim(ids, new)
        same(c, m, str(ids))
        assert m.counts_hold()


def test_trim_into_a_shared_page_then_write(gpu_lib):
    """A sequence cut inside a page that a fork names copies it before it writes there."""
    c, m = pair()
    grow(c, m, [0], [48])
    c.fork(ints([0]), ints([1]))
    m.fork([0], [1])
    c.trim(ints([1]), ints([21]))
    m.trim([1], [21])
    grow(c, m, [1], [30], seed=4)
    same(c, m)
    assert m.tables[0][:3] == [0, 1, 2] and m.tables[1][0] == 0 and m.tables[1][1] != 1 and m.counts_hold()


def test_reserve_refusals(gpu_lib):
    c, m = pair(pages=10, seqs=6, max_pages=4)
    # 0: too long; 1: served; 1 again; bad ids; zero and negative counts; 2: served; 3: past the pages; 4: small, but behind 3
    ids, counts = [0, 1, 1, -1, 6, 5, 5, 2, 3, 4], [65, 64, 1, 1, 1, 0, -3, 40, 64, 1]
    assert grow(c, m, ids, counts) == [0, 64, 0, 0, 0, 0, 0, 40, 0, 0]
    same(c, m)
    # without a new page an entry is served though an earlier one was refused
    assert grow(c, m, [3, 2, 4], [64, 8, 16], seed=2) == [0, 8, 0]
    assert grow(c, m, [4, 3], [16, 32], seed=3) == [16, 32]
    same(c, m)
    assert sum(r == 0 for r in m.refs) == 0
    assert grow(c, m, [4, 5], [1, 1]) == [0, 0]
    same(c, m)


def test_refused_copy_changes_nothing(gpu_lib):
    c, m = pair(pages=2)
    grow(c, m, [0], [20])
    c.fork(ints([0]), ints([1]))
    m.fork([0], [1])
    assert grow(c, m, [1], [1]) == [0]
    same(c, m)


@pytest.mark.parametrize("n,pages,kv,d", [(1024, 3000, 1, 64), (1000, 1500, 2, 96), (1024, 2047, 1, 64)])
def test_many_entries(gpu_lib, n, pages, kv, d):
    """As many entries as a call takes, with the pool running out among them."""
    rng = random.Random(n + pages)
    c, m = pair(pages=pages, kv=kv, d=d, seqs=n + 5, max_pages=5)
    ids = rng.sample(range(n + 5), n)
    grow(c, m, ids, [rng.choice((1, 15, 16, 17, 33, 80, 81)) for _ in ids])
    same(c, m)
    keep = rng.sample(ids, n // 2)
    c.trim(ints(keep), ints([rng.randint(0, 40) for _ in keep]))
    rng = random.Random(n + pages)                    # the same draws for the model
    ids2 = rng.sample(range(n + 5), n)
    [rng.choice((1, 15, 16, 17, 33, 80, 81)) for _ in ids2]
    keep2 = rng.sample(ids2, n // 2)
    m.trim(keep2, [rng.randint(0, 40) for _ in keep2])
    same(c, m)
    assert int(c.compact().item()) == m.compact()
    same(c, m)
    assert m.counts_hold()


@pytest.mark.parametrize("pages", [1, 63, 64, 65, 1023, 1024, 1025, 8193, 70000])
def test_free_pages_in_order(gpu_lib, pages):
    """The lowest free pages go out first, whatever the pool's size, and compaction fills the lowest holes."""
    rng = random.Random(pages)
    c, m = pair(pages=pages, page=16, kv=1, d=64, seqs=4, max_pages=max(pages, 2))
    held = [p for p in range(pages) if rng.random() < 0.5]
    row = held + [-1] * (max(pages, 2) - len(held))
    rng.shuffle(held)
    row[:len(held)] = held
    m.tables[2], m.lens[2] = list(row), 16 * len(held)
    for p in held:
        m.refs[p] = 1
    c.tables[2].copy_(ints(row))
    c.lens[2] = 16 * len(held)
    c.refs.copy_(ints(m.refs))
    n = pages - len(held)
    granted = c.reserve(ints([0, 1]), ints([16 * (n // 3) + 1, 16 * (n // 3)]))
    assert granted.cpu().tolist() == m.reserve([0, 1], [16 * (n // 3) + 1, 16 * (n // 3)])
    same(c, m)
    c.trim(ints([0]))
    m.trim([0])
    assert int(c.compact().item()) == m.compact()
    same(c, m)


def test_append_ragged_and_skipped(gpu_lib):
    """Rows past an entry's count, entries of count 0 and foreign ids are not written."""
    c, m = pair(layers=2, page=32, d=96, kv=5)
    grow(c, m, [0, 1, 2], [40, 3, 70])
    k, v = kv_rows(c, 6, 70, 11)
    ids, counts = [0, 5, 1, 2, 9, -2], [40, 4, -3, 71, 5, 5]
    c.append(1, k.cuda().view(torch.bfloat16), v.cuda().view(torch.bfloat16), ints(ids), ints(counts))
    m.append(1, k.numpy(), v.numpy(), ids, counts)
    same(c, m)


def test_shared_pages(gpu_lib):
    c, m = pair(pages=600, seqs=9, max_pages=200)
    grow(c, m, [0], [16 * 150 + 3])
    c.fork(ints([0] * 4), ints([1, 2, 3, 4]))
    m.fork([0] * 4, [1, 2, 3, 4])
    c.trim(ints([2, 3]), ints([16 * 64, 16 * 65 + 1]))
    m.trim([2, 3], [16 * 64, 16 * 65 + 1])
    grow(c, m, [1, 2, 3, 5], [30, 30, 5, 7], seed=8)
    for ids in ([0, 1, 2, 3, 4, 5, 6], [5, 0, 0, 4, 9, 1, -1, 3, 2], [3]):
        for least in (1, 64, 65, 151):
            assert c.shared(ints(ids), least).cpu().tolist() == m.shared(ids, least), (ids, least)
    assert c.shared().cpu().tolist() == m.shared(list(range(9)))


def test_no_entries(gpu_lib):
    c, m = pair()
    grow(c, m, [0], [5])
    c.trim(ints([]))
    assert c.fork(ints([]), ints([])).numel() == c.reserve(ints([]), ints([])).numel() == 0
    same(c, m)


@pytest.mark.parametrize("seed", range(6))
def test_random_runs(gpu_lib, seed):
    """Forks, growth, trims and compactions in any order, entries refused among them."""
    rng = random.Random(seed)
    page, d, kv = rng.choice((16, 32, 64, 128)), rng.choice((64, 96, 128)), rng.choice((1, 2, 7))
    c, m = pair(layers=rng.choice((1, 3)), pages=rng.randint(8, 90), page=page, kv=kv, d=d, seqs=12, max_pages=rng.randint(2, 9), seed=seed)
    say(f"random run {seed}: page {page} d {d} kv {kv} pages {m.pages} columns {m.max_pages}")
    for step in range(40):
        n = rng.randint(1, 10)
        ids = [rng.randint(-1, 12) for _ in range(n)]
        op = rng.choice(("fork", "grow", "grow", "trim", "compact", "shared"))
        if op == "fork":
            dst = [rng.randint(-1, 12) for _ in range(n)]
            assert c.fork(ints(ids), ints(dst)).cpu().tolist() == m.fork(ids, dst)
        elif op == "grow":
            grow(c, m, ids, [rng.choice((0, 1, 2, page, rng.randint(1, 3 * page))) for _ in ids], seed=step)
        elif op == "trim":
            new = None if rng.random() < 0.3 else [rng.randint(-1, 4 * page) for _ in ids]
            c.trim(ints(ids), None if new is None else ints(new))
            m.trim(ids, new)
        elif op == "compact":
            assert int(c.compact().item()) == m.compact()
        else:
            assert c.shared(ints(ids)).cpu().tolist() == m.shared(ids)
        same(c, m, f"step {step}: {op}")
        assert m.counts_hold()


def test_a_step_in_a_graph(gpu_lib):
    """Free, fork, reserve and append captured once: every replay gives the eager state."""
    c, m = pair(layers=2)
    grow(c, m, [0, 1], [20, 35])
    src, dst, counts = ints([0, 1, 1]), ints([2, 3, 4]), ints([1, 17, 3])
    done, granted = torch.empty_like(src), torch.empty_like(src)
    k, v = kv_rows(c, 3, 17, 21)
    kd, vd = k.cuda().view(torch.bfloat16), v.cuda().view(torch.bfloat16)

    def step():
        c.trim(dst)
        c.fork(src, dst, done)
        c.reserve(dst, counts, granted)
        for layer in range(2):
            c.append(layer, kd, vd, dst, granted)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        graph.replay()
        m.trim([2, 3, 4])
        m.fork([0, 1, 1], [2, 3, 4])
        want = m.reserve([2, 3, 4], [1, 17, 3])
        for layer in range(2):
            m.append(layer, k.numpy(), v.numpy(), [2, 3, 4], want)
        same(c, m, f"replay {rep}")
        assert granted.cpu().tolist() == want
        if rep % 2:
            grow(c, m, [0], [1], seed=rep)            # eager work between replays
            same(c, m)


def test_binding_functions(gpu_lib):
    """The binding's functions, one per C entry point, on the caller's own buffers and on a stream that is passed in."""
    w = gpu_lib
    c = w.make_cache(30, 16, 2, 64, 2, 6, 8)
    m = Model(2, 30, 16, 2, 64, 6, 8, np.zeros((2, 30, 2, 16, 64), np.int16))
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        pool = torch.zeros((2, 30, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
        tables, lens, refs = torch.full((6, 8), -1, dtype=torch.int32, device="cuda"), ints([0] * 6), ints([0] * 30)
        ws = torch.empty(w.wise_cache_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        a = w.make_queries(2, 4)
        aws = torch.empty(w.wise_prefix_workspace_bytes(c, a), dtype=torch.uint8, device="cuda")
        granted, done, shared, live = ints([0] * 2), ints([0] * 2), ints([0] * 2), ints([0])
        k, v = (torch.randint(-2 ** 14, 2 ** 14, (2, 2, 40, 64), dtype=torch.int16, generator=torch.Generator().manual_seed(i)) for i in (1, 2))
        kd, vd, q = k.cuda().view(torch.bfloat16), v.cuda().view(torch.bfloat16), torch.randn(2, 4, 1, 64, device="cuda").to(torch.bfloat16)
        out, lse = torch.empty_like(q), torch.empty((2, 4, 1), device="cuda")
    w.wise_cache_reserve(c, ints([1, 4]), ints([40, 21]), tables, lens, refs, granted, pool, ws, stream=st)
    w.wise_cache_append(c, 40, ints([1, 4]), granted, kd, vd, tables, lens, pool[0], pool[1], stream=st)
    w.wise_cache_fork(c, ints([1, 4]), ints([0, 5]), tables, lens, refs, done, stream=st)
    w.wise_cache_trim(c, ints([4, 1]), ints([0, 17]), tables, lens, refs, stream=st)
    w.wise_cache_compact(c, tables, refs, pool, live, ws, stream=st)
    w.wise_cache_shared(c, 2, 1, ints([0, 1]), tables, lens, shared, stream=st)
    w.wise_prefix_attn(c, a, q, pool[0], pool[1], tables, lens, ints([0, 1]), shared, out, lse, aws, stream=st)
    want = m.reserve([1, 4], [40, 21])
    m.append(0, k.numpy(), v.numpy(), [1, 4], want)
    assert m.fork([1, 4], [0, 5]) == [1, 1]
    m.trim([4, 1], [0, 17])
    pages = m.compact()
    st.synchronize()
    assert granted.cpu().tolist() == want and done.cpu().tolist() == [1, 1] and live.cpu().tolist() == [pages]
    assert tables.cpu().tolist() == m.tables and lens.cpu().tolist() == m.lens and refs.cpu().tolist() == m.refs
    assert np.array_equal(bits(pool), m.pool) and shared.cpu().tolist() == m.shared([0, 1]) == [0, 1]
    again = PagedCache(1, 30, 16, 2, 64, 6, 8, pool=pool, tables=tables, lens=lens, refs=refs)
    out2 = again.attend(0, q, torch.empty_like(q), seq_ids=ints([0, 1]), shared=shared)
    # the keys are any bits, NaN among them: the same bits, from the same kernels
    assert np.array_equal(bits(out), bits(out2))
    with pytest.raises(w.WiseError):
        w.wise_prefix_attn(c, a, q, pool[0], pool[1], tables, lens, None, None, out, lse, aws[:256])
    with pytest.raises(w.WiseError):
        w.wise_prefix_attn(c, a, q, pool[0], pool[1], tables, lens, None, None, out, lse, None)
    for bad in (dict(q=q.float()), dict(q=q[:1]), dict(seq_ids=ints([0])), dict(seq_ids=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        args = dict(dict(q=q, seq_ids=ints([0, 1])), **bad)
        with pytest.raises(ValueError):
            w.wise_prefix_attn(c, a, args["q"], pool[0], pool[1], tables, lens, args["seq_ids"], None, out, lse, aws)


def test_paged_cache_arguments(gpu_lib):
    """What PagedCache refuses before any launch: types, sizes, strides, devices, layers."""
    c, m = pair()
    grow(c, m, [0], [20])
    q = torch.zeros((1, 4, 1, 64), dtype=torch.bfloat16, device="cuda")
    good = dict(q=q, out=torch.empty_like(q))
    c.attend(0, **good)
    c.attend(0, q.view(1, 1, 4, 64).transpose(1, 2), good["out"])     # strides of dims of one do not matter
    for bad in (dict(q=q.half()), dict(out=torch.empty_like(q).float()), dict(seq_ids=torch.tensor([0], device="cuda")),
                dict(seq_ids=torch.tensor([0], dtype=torch.int32)), dict(shared=ints([])), dict(lse=torch.empty(4, device="cuda", dtype=torch.float64)),
                dict(lse=torch.empty(3, device="cuda")), dict(q=torch.zeros((1, 4, 1, 128), dtype=torch.bfloat16, device="cuda")[..., ::2])):
        with pytest.raises(ValueError):
            c.attend(0, **dict(good, **bad))
    with pytest.raises(ValueError):
        c.attend(1, **good)
    for call in (lambda: c.fork(ints([0]), ints([])), lambda: c.trim(torch.tensor([0], device="cuda")), lambda: c.reserve(ints([0, 1]), ints([1])),
                 lambda: c.shared(out=ints([0])), lambda: c.append(0, *kv_rows(c, 1, 1, 0), ints([0]), ints([1]))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(gpu_lib.WiseError):
        c.attend(0, torch.zeros((1, 3, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 3, 1, 64), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(gpu_lib.WiseError):
        c.trim(torch.zeros(1025, dtype=torch.int32, device="cuda"))
    same(c, m)


def test_a_step_with_nothing_to_do(gpu_lib):
    """Every call of a serving step takes an empty batch, still checks its arguments, and changes nothing."""
    c, m = pair()
    grow(c, m, [0], [20])
    none = ints([])
    k = torch.empty((0, 2, 0, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.empty((0, 4, 1, 64), dtype=torch.bfloat16, device="cuda")
    c.trim(none, none)
    assert c.fork(none, none).numel() == 0 and c.reserve(none, none).numel() == 0
    c.append(0, k, k, none, none)
    shared = c.shared(none)
    assert shared.shape == (0,) and shared.dtype == torch.int32
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    assert c.attend(0, q, out, lse, seq_ids=none, shared=shared) is out
    same(c, m)
    for call in (lambda: c.shared(torch.empty(0, device="cuda")), lambda: c.attend(0, q, out.float()), lambda: c.attend(1, q, out),
                 lambda: c.append(0, k.half(), k.half(), none, none), lambda: c.append(1, k, k, none, none)):
        with pytest.raises(ValueError):
            call()
