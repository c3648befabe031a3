"""wise_qcache_attn on the GPU in the paths that large calls take: even shares of many long sequences, pieces of many rows over
thousands of keys, values at the borders of fp16, and tables with room, which are cut and joined where tight ones are not."""

import random

import numpy as np
import pytest
import torch

from kept_model import pack, page_bytes, places, unpack
from paper_2609_27373_amd import wise
from paper_2609_27373_amd.cache import PagedCache, QuantCache
from parity_util import say
from test_gpu_qprefix import Batch, WIDTHS, ints

pytestmark = pytest.mark.gpu

WHOLE = 2560                                          # tokens of a table from which on no call is done uncut


def tokens(cache):
    return cache.shape.max_pages * cache.shape.page


# (sequences, page, head_dim, key-value heads, query heads of each, q_len, bits): up to 8, 16 and 32 rows.
@pytest.mark.parametrize("batch,page,d,kv,gq,q_len,bits", [(64, 16, 64, 2, 4, 1, 4), (65, 32, 128, 1, 1, 1, 8), (128, 16, 96, 1, 8, 2, 4),
                                                           (256, 64, 64, 1, 7, 1, 8), (256, 32, 64, 1, 2, 4, 4), (20, 16, 128, 2, 20, 1, 8),
                                                           (65, 16, 96, 1, 8, 3, 4), (256, 32, 64, 1, 32, 1, 8)])
@pytest.mark.parametrize("prefix", [0, 640])
def test_even_shares_of_many(gpu_lib, batch, page, d, kv, gq, q_len, prefix, bits):
    """64 to 256 sequences of more than 1024 tokens on average, one to 32 rows each, with and without shared pages of up to 32 rows."""
    rng = random.Random(batch + gq)
    rows = gq * q_len
    groups, left = [], batch
    while left:
        n = min(left, rng.randint(1, max(1, 32 // rows)) if prefix else 1)
        groups.append((prefix // page if n > 1 else 0, [rng.choice((1, q_len, 700, 1300, 1900, 2500)) + 500 for _ in range(n)]))
        left -= n
    groups[0] = (groups[0][0], [4000] + groups[0][1][1:])
    groups[-1] = (groups[-1][0], groups[-1][1][:-1] + [None if groups[-1][0] == 0 else 9])
    b = Batch(groups, page, d, kv, gq, bits, q_len, seed=batch, slots=True)
    keys = sum(pre * page + sum(x or 0 for x in tails) for pre, tails in groups)      # shared pages once
    assert tokens(b.cache) > WHOLE and batch <= 256 and rows <= 32 and keys >= 1024 * batch
    say(f"{batch} sequences, {keys} keys, {rows} rows, d {d}, bits {bits}")
    truth = b.truth()
    for shared in (True, False):
        b.check(*b.run(shared), truth)


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
def test_more_than_256_sequences_of_some_length(gpu_lib, d, bits):
    """A plan of its own launch, pieces of all kinds."""
    rng = random.Random(d)
    b = Batch([(40, [rng.choice((1, 20, 130)) for _ in range(40)]), (0, [rng.randint(1, 400) for _ in range(220)]), (30, [5, 2000, 90])], 16, d, 2, 2,
              bits, 1, seed=d)
    assert tokens(b.roomy()) > WHOLE
    truth = b.truth()
    for shared in (True, False):
        b.check(*b.run(shared, cache=b.roomy()), truth)


def kept(pages, kv, page, d, bits, g):
    """Random pages of one layer on the GPU: any code but NaN, scales of 2^-2 to 2^1."""
    pool = torch.randint(0, 256, (2, pages, kv, page_bytes(page, d, bits)), generator=g, device="cuda", dtype=torch.uint8)
    if bits == 8:
        pool[(pool & 127) == 127] = 1
    at = page * d * bits // 8
    pool[..., at:] = torch.randint(125, 129, pool[..., at:].shape, generator=g, device="cuda", dtype=torch.uint8)
    return pool


def reference_on_gpu(q, k, v):
    """kept_model.attend of one sequence's newest token on the GPU: q [gq][d], k and v [n][d]."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = k.shape
    scale = float(np.float32(1 / np.sqrt(d)))
    x = scale * (q @ k.t().contiguous())
    z = torch.logsumexp(x, -1, keepdim=True)
    p = torch.exp(x - z)
    o, a = p @ v, p @ v.abs()
    e = scale * d * 2.0 ** -24 * (q.abs() @ k.abs().t().contiguous()).amax(-1, keepdim=True)
    extra = 2.0 ** -12 + 2 * e + 2.0 ** -18 + n * 2.0 ** -24
    bound = 2.0 ** -8 * o.abs() + (1 + 2.0 ** -8) * (extra * a + n * 2.0 ** -31 * v.abs().amax())
    return o, z[:, 0], bound, e[:, 0] + 2.0 ** -18 + n * 2.0 ** -24 + 2.0 ** -22 * z[:, 0].abs()


@WIDTHS
@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("batch,kv,gq,page,d,total", [(1, 16, 2, 128, 64, 300001), (1, 1, 1, 16, 128, 700000), (128, 8, 4, 64, 64, 40000),
                                                      (128, 8, 4, 32, 128, 40000), (64, 8, 8, 16, 96, 40000)])
def test_pieces_of_more_than_4096_keys(gpu_lib, batch, kv, gq, page, d, total, far, bits):
    """So many keys that a piece is longer than the page ids that a wave holds at once, for one sequence and shared by many rows;
    with a value past fp16 in one token, whose pieces are streamed."""
    g = torch.Generator(device="cuda").manual_seed(batch)
    cols = -(-total // page)
    n = total // page * page                          # shared by all; each has up to a page of its own
    say(f"{batch} sequences over {total} tokens, {kv} heads of {d}, {bits} bits, far {far}")
    pool = kept(cols + batch, kv, page, d, bits, g)
    order = torch.randperm(cols + batch, generator=g, device="cuda").to(torch.int32)
    tables = order[:cols][None].repeat(batch, 1)
    tables[:, n // page:] = order[cols:cols + batch, None]
    tables = tables[:, :cols].contiguous()
    if far:
        pool[1, int(tables[0, (n // page) // 2]), :, page * d * bits // 8] = 127 + 12
    c = QuantCache(1, cols + batch, page, kv, d, batch, tables.shape[1], bits=bits, pool=pool, tables=tables,
                   lens=torch.full((batch,), total, dtype=torch.int32, device="cuda"))
    q = torch.randn((batch, kv * gq, 1, d), generator=g, device="cuda").to(torch.bfloat16)
    shared = torch.full((batch,), n // page, dtype=torch.int32, device="cuda")
    shared[0] = 0
    if batch > 1:                                     # what a piece of many rows has, by the plan: 256 of them
        assert batch * gq > 64 and -(-batch * gq // 128) * n * kv / 256 > 4096
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    c.attend(0, q, out, lse, shared=shared if batch > 1 else None)
    k, v = (torch.empty((2, kv, total, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    which = sorted({0, batch - 1})
    c.read(0, k[:len(which)], v[:len(which)], ints(which), ints([total] * len(which)))
    for i, b in enumerate(which):
        for h in sorted({0, kv - 1}):
            rows = slice(h * gq, (h + 1) * gq)
            o, z, bound, zb = reference_on_gpu(q[b, rows, 0], k[i, h], v[i, h])
            assert ((out[b, rows, 0].double() - o).abs() <= bound).all()
            assert ((lse[b, rows, 0].double() - z).abs() <= zb).all()


KINDS = {"own": ([(0, [300, 33, 64])], 2, 4, 1), "own, 20 rows": ([(0, [300, 33])], 1, 20, 1), "few": ([(20, [40, 5, 70])], 2, 4, 2),
         "many": ([(40, [30] * 10)], 2, 8, 2)}


@WIDTHS
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("codes", ["all", "least"])
def test_borders_of_fp16(gpu_lib, kind, d, codes, bits):
    """Values at the least and largest scale that fp16 takes, where every product is one of its subnormal numbers or near its largest, and at the next
    ones, which bf16 takes; in all places, and in one token's 32 dims alone."""
    groups, kv, gq, q_len = KINDS[kind]
    b = Batch(groups, 16, d, kv, gq, bits, q_len, seed=d)
    rng = np.random.default_rng(d)
    was, scales = unpack(b.pool[1], 16, d, bits, 1)
    live = scales != 255
    # Of 4 bits every code times 2^-23 is a subnormal number of fp16; of 8 the first eight times 2^-15 are.
    magnitude = rng.integers(0, {"all": {4: 8, 8: 127}, "least": {4: 8, 8: 8}}[codes][bits], was.shape)
    new = np.where(live.repeat(32, -1), magnitude | rng.integers(0, 2, was.shape) << (bits - 1), was).astype(np.uint8)
    least, most = (-23, 8) if bits == 4 else (-15, 7)
    one = tuple(np.argwhere(live)[len(np.argwhere(live)) // 2])
    for e, single in [(e, s) for e in (least - 1, least, most, most + 1) for s in (False, True)]:
        new_scales = np.where(live, 127 if single else 127 + e, 255).astype(np.uint8)
        if single:
            new_scales[one] = 127 + e
        pool = b.pool.copy()
        pool[1] = pack(new, new_scales, bits, 1)
        b.set_pool(pool, 16, d, bits)
        b.cache.pool.copy_(torch.tensor(pool))
        truth = b.truth()
        say(f"2^{e}, one scale {single}, d {d}, bits {bits}, {kind}, codes {codes}")
        for cache in (b.cache, b.roomy()):
            for shared in (True, False):
                b.check(*b.run(shared, cache=cache), truth)


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("members", [3, 40])
def test_nan_codes_in_cut_tables(gpu_lib, d, members):
    """A code that is NaN in shared pages (of few rows, and of many), in a draft's own value, and in a tail: its dim alone."""
    page, q_len, bits = 16, 2, 8
    b = Batch([(40, [20] * members)], page, d, 2, 2, bits, q_len, seed=d)
    o, _, bound, _ = b.truth()
    want, pool = o.copy(), b.pool.copy()
    code = places(page, d, bits, 1)[0]
    for s, pos, h, dim in [(0, 100, 1, d - 1), (0, 639, 0, 0), (1, 640 + 19, 0, 5), (2, 640 + 3, 1, 0)]:
        pool[1, b.tables[s, pos // page], h, code[pos % page, dim]] = 255
        for e in range(members) if pos < 640 else [s]:
            for r in range(q_len):
                if pos <= 660 - q_len + r:
                    want[e, 2 * h:2 * h + 2, r, dim] = np.nan
    b.cache.pool.copy_(torch.tensor(pool))
    for shared in (True, False):
        got = b.run(shared, cache=b.roomy())[0].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        assert np.all(np.abs(got - want)[ok] <= bound[ok])


@WIDTHS
@pytest.mark.parametrize("members", [3, 40])
def test_nan_and_infinite_queries_in_cut_tables(gpu_lib, members, bits):
    """They reach their own row only, also among the many rows of shared pages."""
    b = Batch([(24, [30 + i for i in range(members)])], 32, 64, 2, 2, bits, 2, seed=1)
    truth = b.truth()
    b.q[0, 1, 0, 3] = float("nan")
    b.q[2, 3, 1, 60] = float("inf")
    bad = np.zeros(b.q.shape, bool)
    bad[0, 1, 0] = bad[2, 3, 1] = True
    for shared in (True, False):
        out, lse = b.run(shared, cache=b.roomy())
        got = out.double().cpu().numpy()
        assert np.isnan(got[bad]).all() and np.all(np.abs(got - truth[0])[~bad] <= truth[2][~bad])


@WIDTHS
@pytest.mark.parametrize("members", [1, 14, 60])
def test_two_runs_of_cut_tables_are_equal(gpu_lib, members, bits):
    b = Batch([(20, [30, 400, 1] * members)], 32, 128, 2, 4, bits, 2, seed=5)
    cache = b.roomy()
    first = b.run(cache=cache)
    b.check(*first, b.truth())
    for _ in range(3):
        again = b.run(cache=cache)
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16)) and torch.equal(first[1], again[1])


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("members", [1, 12, 40])
def test_as_the_cache_in_bf16_in_cut_tables(gpu_lib, d, members, bits):
    """PagedCache over the values that read() gives back, both against the definition."""
    page = 32
    b = Batch([(20, [100 + 3 * i for i in range(members)])], page, d, 2, 4, bits, 2, seed=d)
    cache = b.roomy()
    c = cache.shape
    k, v = (torch.zeros((c.seqs, c.kv_heads, int(b.lens.max()), d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.read(0, k, v, ints(range(c.seqs)), cache.lens)
    wide = PagedCache(1, c.pages, page, c.kv_heads, d, c.seqs, c.max_pages, tables=cache.tables.clone(), lens=cache.lens.clone())
    wide.append(0, k, v, ints(range(c.seqs)), cache.lens)
    truth = b.truth()
    for shared in (True, False):
        b.check(*b.run(shared, cache=wide), truth)
        b.check(*b.run(shared, cache=cache), truth)


@WIDTHS
@pytest.mark.parametrize("members", [2, 40])
def test_offsets_past_32_bits_in_cut_tables(gpu_lib, members, bits):
    """Pages that begin behind 4 GiB of a plane, shared by few rows and by many."""
    d, page, kv = 128, 128, 2
    size = page_bytes(page, d, bits)
    pages = (1 << 32) // (kv * size) + 60
    if torch.cuda.mem_get_info()[0] < 3 * pages * kv * size:
        pytest.skip("too little memory")
    b = Batch([(6, [200] * members)], page, d, kv, 4, bits, seed=2)
    cache = b.roomy()
    c = cache.shape
    pool = torch.zeros((2, pages, kv, size), dtype=torch.uint8, device="cuda")
    shift = pages - c.pages
    pool[:, shift:] = cache.pool
    tables = torch.where(cache.tables >= 0, cache.tables + shift, cache.tables)
    big = QuantCache(1, pages, page, kv, d, c.seqs, c.max_pages, bits=bits, pool=pool, tables=tables, lens=cache.lens)
    truth = b.truth()
    for shared in (True, False):
        b.check(*b.run(shared, cache=big), truth)


def test_binding_function_in_cut_tables(gpu_lib):
    b = Batch([(9, [30, 400, 1, 77])], 32, 64, 2, 4, 4, seed=6)
    cache = b.roomy()
    c, a = cache.shape, wise.make_queries(4, 8)
    ws = torch.empty(wise.wise_qcache_workspace_bytes(c, 4, a), dtype=torch.uint8, device="cuda")
    q = b.q.cuda()
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    wise.wise_qcache_attn(c, 4, a, q, *cache.layer(0), cache.tables, cache.lens, ints(b.ids), ints(b.shared), o, lse, ws)
    torch.cuda.synchronize()
    b.check(o, lse, b.truth())
