"""wise_qcache_attn on the GPU against the fp64 definition over what the pages hold, row by
row: one to 128 query rows a key-value head, shared and private pages, lengths at page
and tile borders, NaN kept in values and in places that no row sees, both widths."""

import random

import numpy as np
import pytest
import torch

from cache_model import bf16_values, up
from kept_model import attend, pack, page_bytes, quantise, read_pool
from paper_2609_27373_amd import wise
from paper_2609_27373_amd.cache import PagedCache, QuantCache
from parity_util import say

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Batch:
    """A cache whose unused bytes are 255 (NaN, code and scale), and a batch of queries.  groups: list of (pages shared, [tail
    lengths]); a tail of None is an empty sequence."""

    def __init__(self, groups, page, d, kv, gq, bits, q_len=1, seed=0, gain=1.0, slots=False, spare=3, spread=1.0):
        rng, nr = random.Random(seed), np.random.default_rng(seed)
        batch = sum(len(t) for _, t in groups)
        lens = [0 if x is None else pre * page + x for pre, tails in groups for x in tails]
        need = sum(pre for pre, _ in groups) + sum(up(x or 0, page) for _, t in groups for x in t)
        pages, seqs = need + spare, batch + 2
        cols = max(1, max(up(n, page) for n in lens))
        order = rng.sample(range(pages), pages)
        self.ids = rng.sample(range(seqs), batch) if slots else list(range(batch))
        tables, all_lens, shared, i = np.full((seqs, cols), -1), np.zeros(seqs, int), [], 0
        used = np.zeros(pages, int)                  # tokens that a page holds
        for pre, tails in groups:
            first = [order.pop() for _ in range(pre)]
            for j, x in enumerate(tails):
                row = [] if x is None else first + [order.pop() for _ in range(up(x, page))]
                tables[self.ids[i], :len(row)] = row
                all_lens[self.ids[i]] = lens[i]
                for c, p in enumerate(row):
                    used[p] = min(page, lens[i] - c * page)
                shared.append(pre if j else 0)
                i += 1
        # Scales of their own for every 32 dims: a wrong one shows.
        x = nr.standard_normal((2, pages, kv, page, d)) * np.exp(spread * nr.standard_normal((2, pages, kv, page, d // 32))).repeat(32, -1)
        x = bf16_values(torch.tensor(x).to(torch.bfloat16).view(torch.int16).numpy())
        codes, scales = quantise(x, bits)
        empty = np.arange(page) >= used[:, None]
        codes[np.broadcast_to(empty[None, :, None], codes.shape[:4])] = 15 if bits == 4 else 255
        scales[np.broadcast_to(empty[None, :, None], codes.shape[:4])] = 255
        self.set_pool(np.stack([pack(codes[p], scales[p], bits, p) for p in (0, 1)]), page, d, bits)
        self.tables, self.lens, self.shared = tables, all_lens, shared
        self.q = torch.tensor(gain * nr.standard_normal((batch, kv * gq, q_len, d))).to(torch.bfloat16)
        self.cache = QuantCache(1, pages, page, kv, d, seqs, cols, bits=bits, pool=torch.tensor(self.pool).cuda(), tables=ints(tables.tolist()),
                                lens=ints(all_lens.tolist()))

    def set_pool(self, pool, page, d, bits):
        self.pool, self.page, self.bits = pool, page, bits
        self.k, self.v = read_pool(pool, page, d, bits)

    def roomy(self):
        """The same cache with tables of more than 2560 tokens, which are cut and joined however few sequences hold."""
        c = self.cache.shape
        cols = max(c.max_pages, 2560 // c.page + 2)
        tables = torch.full((c.seqs, cols), -1, dtype=torch.int32, device="cuda")
        tables[:, :c.max_pages] = self.cache.tables
        return QuantCache(1, c.pages, c.page, c.kv_heads, c.head_dim, c.seqs, cols, bits=self.bits, pool=self.cache.pool, tables=tables,
                          lens=self.cache.lens.clone())

    def run(self, shared=True, scale=0.0, out=None, cache=None):
        q = self.q.cuda()
        out = torch.full_like(q, float("nan")) if out is None else out
        lse = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device="cuda")
        (cache or self.cache).attend(0, q, out, lse, seq_ids=ints(self.ids), shared=ints(self.shared) if shared else None, scale=scale)
        torch.cuda.synchronize()
        return out, lse

    def truth(self, scale=0.0):
        q = bf16_values(self.q.view(torch.int16).numpy())
        scale = np.float32(scale if scale > 0 else 1 / np.sqrt(self.q.shape[-1])).astype(float)
        return attend(q, self.k, self.v, self.tables, self.lens, self.ids, self.page, scale)

    def check(self, out, lse, truth):
        o, z, bound, zb = truth
        got, gz = out.float().cpu().numpy().astype(float), lse.cpu().numpy().astype(float)
        err = np.abs(got - o)
        assert np.all(err <= bound), f"o: {np.nanmax(err - bound):.3g} past the bound, NaN {np.isnan(got).sum()}"
        empty = np.isneginf(z)
        assert np.array_equal(np.isneginf(gz), empty)
        assert np.all(np.abs(gz[~empty] - z[~empty]) <= zb[~empty])
        assert np.all(got[empty] == 0)

    def both(self, scale=0.0):
        long = bool((self.lens > self.tables.shape[1] * self.page).any())      # cut by the table itself
        truth = self.truth(scale)
        for cache in (self.cache,) if long else (self.cache, self.roomy()):
            for shared in (True, False):
                self.check(*self.run(shared, scale, cache=cache), truth)


WIDTHS = pytest.mark.parametrize("bits", [4, 8])


@WIDTHS
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("gq", [1, 4, 7])
def test_lengths(gpu_lib, page, d, gq, bits):
    """No prefix: empty, one token, and every side of the page and tile borders."""
    tails = [None, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 300]
    Batch([(0, tails)], page, d, 2, gq, bits, seed=page + d + gq).both()


@WIDTHS
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("gq", [1, 4, 8, 9, 20])
def test_lengths_beside_a_long_one(gpu_lib, page, d, gq, bits):
    """The same where sequences are cut and joined: a table of more than 512 tokens."""
    tails = [None, 1, 16, 17, 63, 64, 65, 127, 128, 129, 256, 257, 1500, 33, None, 700]
    Batch([(0, tails)], page, d, 2, gq, bits, seed=page + d + gq).both()


@WIDTHS
@pytest.mark.parametrize("batch", [63, 65, 128, 256, 257])
def test_batch_sizes(gpu_lib, batch, bits):
    """Runs that cross the 64 sequences of a planning wave and the 256 of a work-group's own plan."""
    rng = random.Random(batch)
    groups, left = [], batch
    while left:
        n = min(left, rng.choice((1, 2, 30, 70)))
        groups.append((rng.choice((4, 9, 44)) if n > 1 else 0, [rng.choice((None, 1, 20, 50)) if n < 30 else rng.randint(1, 50) for _ in range(n)]))
        left -= n
    Batch(groups, 16, 64, 2, 2, bits, seed=batch, slots=True).both()


@WIDTHS
@pytest.mark.parametrize("d,kv,gq,q_len", [(64, 5, 1, 1), (96, 3, 4, 3), (128, 8, 5, 4)])
@pytest.mark.parametrize("longest", [100, 400, 2000])
def test_more_heads_than_groups(gpu_lib, d, kv, gq, q_len, longest, bits):
    """So many sequences and heads that short tails are a wave's each; heads that 4 does not divide."""
    rng = random.Random(d + kv)
    tails = [rng.choice((None, 1, 2, q_len, 31, 32, 33, 64, 100, 127, 128, 129, 160)) for _ in range(600 // kv)]
    tails = [x if x is None else min(x, longest) for x in tails] + [longest]
    Batch([(0, tails[:40]), (3, tails[40:60]), (0, tails[60:])], 32, d, kv, gq, bits, q_len, seed=longest).both()


@WIDTHS
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("members", [2, 17, 40])
def test_shared_prefix(gpu_lib, page, d, members, bits):
    """2, 17 and 40 members of four rows: few rows and, from 65 on, many; prefixes of a few tiles."""
    rng = random.Random(members)
    Batch([(320 // page + 3, [rng.choice((1, 3, 50, 130)) for _ in range(members)])], page, d, 2, 4, bits, seed=members).both()


@WIDTHS
@pytest.mark.parametrize("gq,q_len", [(1, 2), (1, 128), (4, 5), (8, 4), (8, 16), (3, 11), (128, 1), (16, 2), (33, 1), (17, 3), (8, 1), (2, 4), (9, 1)])
@pytest.mark.parametrize("d,page", [(64, 16), (96, 64), (128, 32)])
def test_query_rows(gpu_lib, gq, q_len, d, page, bits):
    """Every number of row tiles, drafts causal among themselves, with and without shared pages."""
    tails = [x + q_len for x in (0, 1, 30, 64, 200)]
    Batch([(256 // page, tails), (0, tails[:3])], page, d, 2, gq, bits, q_len, seed=gq + q_len).both()


@WIDTHS
@pytest.mark.parametrize("d,page", [(64, 32), (96, 16), (128, 128)])
def test_drafts_longer_than_tails(gpu_lib, d, page, bits):
    """Queries of positions before the first: rows that see nothing."""
    Batch([(0, [1, 2, 3, 7, 20, None])], page, d, 2, 4, bits, 7, seed=d).both()


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("kv,gq", [(1, 1), (5, 1), (2, 8)])
def test_long(gpu_lib, d, kv, gq, bits):
    """Many pieces a row, page ids reloaded on the way."""
    Batch([(0, [9001, 33, 5000])], 16, d, kv, gq, bits, seed=d).both()


@WIDTHS
@pytest.mark.parametrize("page,d,kv,gq,q_len", [(16, 64, 2, 4, 1), (128, 128, 3, 1, 1), (32, 96, 1, 8, 2), (64, 128, 11, 1, 1)])
@pytest.mark.parametrize("groups", [[(0, [1500, None, 2500, 900, 33, 4000])], [(40, [700, 1, 2100]), (0, [1900, 1300]), (70, [20, 1000, 9])],
                                    [(0, [1200 + 7 * i for i in range(70)])]])
def test_even_shares(gpu_lib, page, d, kv, gq, q_len, groups, bits):
    """Sequences of more than 1024 tokens on average, which are laid one behind another and cut evenly: shared pages too, more
    than 64 sequences, numbers of heads that the work-groups do not divide."""
    if kv == 11 and len(groups[0][1]) > 10:
        groups = [(0, groups[0][1][:9])]
    groups = [(pre * 16 // page, tails) for pre, tails in groups]
    b = Batch(groups, page, d, kv, gq, bits, q_len, seed=page)
    truth = b.truth()
    for shared in (True, False):
        b.check(*b.run(shared), truth)


@WIDTHS
@pytest.mark.parametrize("gain,scale", [(60.0, 0.0), (1.0, 3.0), (0.0, 0.0), (1.0, 1e-6)])
def test_scores(gpu_lib, gain, scale, bits):
    """Scores so large that one key has all the weight, none at all, and a scale of the caller's."""
    Batch([(8, [50, 300, 1])], 32, 96, 2, 4, bits, seed=3, gain=gain).both(scale)


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
def test_every_scale(gpu_lib, d, bits):
    """Scales from the smallest that is written to the largest whose products stay finite."""
    b = Batch([(0, [500, 70])], 32, d, 2, 2, bits, seed=d)
    page, lo, hi = 32, (2, 252) if bits == 4 else (10, 246), 127 + 100
    nr = np.random.default_rng(1)
    pool = b.pool.copy()
    at = page * d * bits // 8
    live = pool[1][..., at:] != 255
    pool[1][..., at:][live] = nr.integers(lo[0], hi, live.sum())             # values: sums of 2^100 are finite
    live = pool[0][..., at:] != 255
    pool[0][..., at:][live] = nr.integers(lo[0], 128, live.sum())
    b.set_pool(pool, page, d, bits)
    b.cache.pool.copy_(torch.tensor(pool))
    b.both()


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("roomy", [False, True])
def test_nan_values(gpu_lib, d, roomy, bits):
    """A NaN scale of a value makes its 32 dims NaN in the rows that see it and in no other row or dim; a NaN key whole rows."""
    q_len, page, lens = 4, 16, [70, 40, 300]
    b = Batch([(0, lens)], page, d, 2, 2, bits, q_len, seed=d)
    clean = b.truth()
    want = clean[0].copy()
    hit = [(0, 67, 0, 0), (0, 69, 1, d // 32 - 1), (1, 0, 1, 1), (2, 299, 0, 1), (2, 140, 1, 0)]   # sequence, position, head, scale
    pool = b.pool.copy()
    row, g = d * bits // 8, d // 32
    for s, pos, h, i in hit:
        p, t = b.tables[s, pos // page], pos % page
        pool[1, p, h, page * row + t // 4 * 4 * g + 4 * i + t % 4] = 255
        for r in range(q_len):
            if pos <= lens[s] - q_len + r:
                want[s, 2 * h:2 * h + 2, r, 32 * i:32 * i + 32] = np.nan
    key = (1, 38, 0)                                                       # seen by the last two rows
    pool[0, b.tables[1, key[1] // page], key[2], page * row + key[1] % page * g] = 255
    b.cache.pool.copy_(torch.tensor(pool))
    out, lse = b.run(cache=b.roomy() if roomy else None)
    got, gz = out.double().cpu().numpy(), lse.double().cpu().numpy()
    want[1, :2, 2:] = np.nan
    assert np.isnan(gz[1, :2, 2:]).all()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.all(np.abs(got - want)[ok] <= clean[2][ok])


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("members", [3, 40])
def test_nan_codes(gpu_lib, d, members):
    """A code that is NaN (E4M3 has one) in shared pages, in a draft's own key, and in a tail: its dim alone."""
    page, q_len, bits = 16, 2, 8
    b = Batch([(16, [20] * members)], page, d, 2, 2, bits, q_len, seed=d)
    o, _, bound, _ = b.truth()
    want, pool = o.copy(), b.pool.copy()
    from kept_model import places
    code = places(page, d, bits, 1)[0]
    for s, pos, h, dim in [(0, 100, 1, d - 1), (1, 256 + 19, 0, 5), (2, 256 + 3, 1, 0)]:
        pool[1, b.tables[s, pos // page], h, code[pos % page, dim]] = 127
        for e in range(members) if pos < 256 else [s]:
            for r in range(q_len):
                if pos <= 276 - q_len + r:
                    want[e, 2 * h:2 * h + 2, r, dim] = np.nan
    b.cache.pool.copy_(torch.tensor(pool))
    for shared in (True, False):
        got = b.run(shared)[0].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        assert np.all(np.abs(got - want)[ok] <= bound[ok])


@WIDTHS
def test_nan_and_infinite_queries(gpu_lib, bits):
    """They reach their own row only."""
    b = Batch([(8, [30, 40, 50])], 32, 64, 2, 2, bits, 2, seed=1)
    truth = b.truth()
    b.q[0, 1, 0, 3] = float("nan")
    b.q[2, 3, 1, 60] = float("inf")
    out, lse = b.run()
    got = out.double().cpu().numpy()
    bad = np.zeros(got.shape, bool)
    bad[0, 1, 0] = bad[2, 3, 1] = True
    assert np.isnan(got[bad]).all() and np.all(np.abs(got - truth[0])[~bad] <= truth[2][~bad])


@WIDTHS
@pytest.mark.parametrize("d", [64, 128])
def test_bad_tables_and_lengths(gpu_lib, d, bits):
    """Page ids out of range are not followed (their positions are not attended), lengths past the table are cut to it."""
    b = Batch([(0, [200, 90, 64, 33])], 16, d, 2, 3, bits, 2, seed=9)
    for s, j, v in [(0, 3, -1), (0, 4, 1 << 30), (1, 0, -7), (2, 0, b.cache.shape.pages), (2, 1, -1), (2, 2, -1), (2, 3, -1)]:
        b.tables[s, j] = v
    b.cache.tables.copy_(ints(b.tables.tolist()))
    b.both()
    b.lens[0] = 1 << 20
    b.lens[3] = -5
    b.tables[0] = b.tables[0].clip(0, b.cache.shape.pages - 1)
    pool = b.pool.copy()
    at = 16 * d * bits // 8
    pool[..., at:][pool[..., at:] == 255] = 127
    pool[..., :at][pool[..., :at] == 255] = 0
    b.set_pool(pool, 16, d, bits)
    b.cache.pool.copy_(torch.tensor(pool))
    b.cache.tables.copy_(ints(b.tables.tolist()))
    b.cache.lens.copy_(ints(b.lens.tolist()))
    b.check(*b.run(False), b.truth())


@WIDTHS
@pytest.mark.parametrize("members", [3, 40])
def test_bad_page_shared_by_many(gpu_lib, members, bits):
    b = Batch([(20, [5] * members)], 16, 128, 2, 4, bits, seed=members)
    b.tables[:members, 7] = -1
    b.cache.tables.copy_(ints(b.tables.tolist()))
    b.both()


@WIDTHS
def test_repeated_and_foreign_ids(gpu_lib, bits):
    b = Batch([(0, [40, 100, 7])], 32, 96, 2, 2, bits, seed=4)
    b.ids = [1, 1, -3]
    b.check(*b.run(False), b.truth())
    b.ids = [0, 99, 0]
    b.check(*b.run(False), b.truth())


@WIDTHS
def test_rows_are_left_alone(gpu_lib, bits):
    """Nothing outside o and lse is written: rows behind the batch keep what they held."""
    b = Batch([(0, [40, 100])], 32, 96, 2, 2, bits, seed=4)
    q = b.q.cuda()
    out = torch.full((3, *q.shape[1:]), 7.0, dtype=torch.bfloat16, device="cuda")
    before = b.cache.pool.clone()
    b.cache.attend(0, q, out[:2], seq_ids=ints(b.ids))
    torch.cuda.synchronize()
    assert (out[2] == 7).all() and torch.equal(before, b.cache.pool)


@WIDTHS
def test_two_runs_are_equal(gpu_lib, bits):
    b = Batch([(20, [30, 400, 1] * 14)], 32, 128, 2, 4, bits, 2, seed=5)
    first = b.run()
    for _ in range(3):
        again = b.run()
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16)) and torch.equal(first[1], again[1])


@WIDTHS
@pytest.mark.parametrize("members", [2, 40])
def test_offsets_past_32_bits(gpu_lib, members, bits):
    """Pages that begin behind 4 GiB of a plane."""
    d, page, kv = 128, 128, 2
    size = page_bytes(page, d, bits)
    pages = (1 << 32) // (kv * size) + 40
    if torch.cuda.mem_get_info()[0] < 3 * pages * kv * size:
        pytest.skip("too little memory")
    b = Batch([(3, [200] * members)], page, d, kv, 4, bits, seed=2)
    small = b.cache.shape.pages
    pool = torch.zeros((2, pages, kv, size), dtype=torch.uint8, device="cuda")
    shift = pages - small
    pool[:, shift:] = b.cache.pool
    tables = torch.where(b.cache.tables >= 0, b.cache.tables + shift, b.cache.tables)
    c = b.cache.shape
    big = QuantCache(1, pages, page, kv, d, c.seqs, c.max_pages, bits=bits, pool=pool, tables=tables, lens=b.cache.lens)
    b.check(*b.run(cache=big), b.truth())


@WIDTHS
def test_graph_and_streams(gpu_lib, bits):
    """Captured on a stream of its own, replayed with eager work between, follows new queries and lengths."""
    b = Batch([(9, [30, 400, 1, 77])], 32, 96, 2, 4, bits, seed=6)
    q, ids, shared = b.q.cuda(), ints(b.ids), ints(b.shared)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
    cache = b.roomy()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        cache.attend(0, q, out, lse, seq_ids=ids, shared=shared)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(0, q, out, lse, seq_ids=ids, shared=shared)
    for i in range(4):
        b.q = torch.randn(b.q.shape).to(torch.bfloat16)
        if i == 2:
            b.lens[b.ids[1]] -= 5
            cache.lens.copy_(ints(b.lens.tolist()))
        q.copy_(b.q)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        b.check(out, lse, b.truth())
        eager = b.run(cache=cache)
        assert torch.equal(eager[0].view(torch.int16), out.view(torch.int16))


@WIDTHS
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("members", [1, 12, 40])
def test_as_the_cache_in_bf16_over_what_was_kept(gpu_lib, d, members, bits):
    """PagedCache over the values that read() gives back: the same but for the order of sums, and both against the definition."""
    page = 32
    b = Batch([(10, [100 + 3 * i for i in range(members)])], page, d, 2, 4, bits, 2, seed=d)
    c = b.cache.shape
    longest = int(b.lens.max())
    k, v = (torch.zeros((c.seqs, c.kv_heads, longest, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    b.cache.read(0, k, v, ints(range(c.seqs)), b.cache.lens)
    wide = PagedCache(1, c.pages, page, c.kv_heads, d, c.seqs, c.max_pages, tables=b.cache.tables.clone(), lens=b.cache.lens.clone())
    wide.append(0, k, v, ints(range(c.seqs)), b.cache.lens)
    truth = b.truth()
    for shared in (True, False):
        b.check(*b.run(shared, cache=wide), truth)
        b.check(*b.run(shared), truth)
    say(f"d {d} members {members} bits {bits}")


def test_binding_function(gpu_lib):
    b = Batch([(9, [30, 400, 1, 77])], 32, 64, 2, 4, 4, seed=6)
    c, a = b.cache.shape, wise.make_queries(4, 8)
    ws = torch.empty(wise.wise_qcache_workspace_bytes(c, 4, a), dtype=torch.uint8, device="cuda")
    q = b.q.cuda()
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    wise.wise_qcache_attn(c, 4, a, q, *b.cache.layer(0), b.cache.tables, b.cache.lens, ints(b.ids), ints(b.shared), o, lse, ws)
    torch.cuda.synchronize()
    b.check(o, lse, b.truth())
    with pytest.raises(ValueError):
        wise.wise_qcache_attn(c, 4, a, q.float(), *b.cache.layer(0), b.cache.tables, b.cache.lens, None, None, o, lse, ws)
