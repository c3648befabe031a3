"""wise_prefix_attn on the GPU against the fp64 definition, row by row: one
to 128 query rows a key-value head, shared and private pages, empty and one-token
sequences, lengths at page and tile borders, garbage beyond a sequence."""

import random

import numpy as np
import pytest
import torch

from cache_model import attend, bf16_values, up
from paper_2609_27373_amd.cache import PagedCache
from parity_util import say

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Batch:
    """A cache whose unused slots hold NaN, and a batch of queries.  groups: list of (pages shared, [tail lengths]);
    a tail of None is an empty sequence."""

    def __init__(self, groups, page, d, kv, gq, q_len=1, seed=0, gain=1.0, slots=False, spare=3):
        g = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        batch = sum(len(t) for _, t in groups)
        lens = [0 if x is None else pre * page + x for pre, tails in groups for x in tails]
        need = sum(pre for pre, _ in groups) + sum(up(x or 0, page) for _, t in groups for x in t)
        pages, seqs = need + spare, batch + 2
        cols = max(1, max(up(n, page) for n in lens))
        order = rng.sample(range(pages), pages)
        self.ids = rng.sample(range(seqs), batch) if slots else list(range(batch))
        tables, all_lens, shared, i = np.full((seqs, cols), -1), np.zeros(seqs, int), [], 0
        for pre, tails in groups:
            first = [order.pop() for _ in range(pre)]
            for j, x in enumerate(tails):
                row = [] if x is None else first + [order.pop() for _ in range(up(x, page))]
                tables[self.ids[i], :len(row)] = row
                all_lens[self.ids[i]] = lens[i]
                shared.append(pre if j else 0)
                i += 1
        pool = torch.full((2, pages, kv, page, d), float("nan"), dtype=torch.bfloat16)
        for s in range(seqs):
            for p0 in range(0, int(all_lens[s]), page):
                n = min(page, int(all_lens[s]) - p0)
                p = int(tables[s, p0 // page])
                if torch.isnan(pool[0, p, 0, 0, 0]):
                    pool[:, p, :, :n] = torch.randn((2, kv, n, d), generator=g).to(torch.bfloat16)
        self.tables, self.lens, self.shared, self.page = tables, all_lens, shared, page
        self.pool = pool
        self.q = (gain * torch.randn((batch, kv * gq, q_len, d), generator=g)).to(torch.bfloat16)
        self.cache = PagedCache(1, pages, page, kv, d, seqs, cols, pool=pool.cuda(), tables=ints(tables.tolist()),
                                lens=ints(all_lens.tolist()))

    def roomy(self):
        """The same cache with tables of more than 2048 tokens, which are cut and joined however few sequences hold."""
        c = self.cache.shape
        cols = max(c.max_pages, 2048 // c.page + 2)
        tables = torch.full((c.seqs, cols), -1, dtype=torch.int32, device="cuda")
        tables[:, :c.max_pages] = self.cache.tables
        return PagedCache(1, c.pages, c.page, c.kv_heads, c.head_dim, c.seqs, cols, pool=self.cache.pool, tables=tables, lens=self.cache.lens.clone())

    def run(self, shared=True, scale=0.0, out=None, cache=None):
        q = self.q.cuda()
        out = torch.full_like(q, float("nan")) if out is None else out
        lse = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device="cuda")
        (cache or self.cache).attend(0, q, out, lse, seq_ids=ints(self.ids), shared=ints(self.shared) if shared else None, scale=scale)
        torch.cuda.synchronize()
        return out, lse

    def check(self, out, lse, scale=0.0):
        f64 = lambda t: bf16_values(t.view(torch.int16).numpy())  # noqa: E731
        scale = np.float32(scale if scale > 0 else 1 / np.sqrt(self.q.shape[-1])).astype(float)
        o, z, bound, zb = attend(f64(self.q), f64(self.pool[0]), f64(self.pool[1]), self.tables, self.lens, self.ids, self.page, scale)
        got, gz = out.float().cpu().numpy().astype(float), lse.cpu().numpy().astype(float)
        err = np.abs(got - o)
        assert np.all(err <= bound), f"o: {np.nanmax(err - bound):.3g} past the bound, NaN {np.isnan(got).sum()}"
        empty = np.isneginf(z)
        assert np.array_equal(np.isneginf(gz), empty)
        assert np.all(np.abs(gz[~empty] - z[~empty]) <= zb[~empty])
        assert np.all(got[empty] == 0)

    def both(self, scale=0.0):
        long = bool((self.lens > self.tables.shape[1] * self.page).any())      # cut by the table itself
        for cache in (self.cache,) if long else (self.cache, self.roomy()):
            for shared in (True, False):
                self.check(*self.run(shared, scale, cache=cache), scale)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("gq", [1, 4, 7])
def test_lengths(gpu_lib, page, d, gq):
    """No prefix: empty, one token, and every side of the page and tile borders."""
    tails = [None, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 300]
    b = Batch([(0, tails)], page, d, 2, gq, seed=page + d + gq)
    b.both()


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("gq", [1, 4, 20])
def test_lengths_beside_a_long_one(gpu_lib, page, d, gq):
    """The same where sequences are cut and joined: a table of more than 512 tokens."""
    tails = [None, 1, 16, 17, 63, 64, 65, 127, 128, 129, 256, 257, 1500, 33, None, 700]
    b = Batch([(0, tails)], page, d, 2, gq, seed=page + d + gq)
    b.both()


@pytest.mark.parametrize("batch", [63, 64, 65, 128, 200, 256, 257])
def test_batch_sizes(gpu_lib, batch):
    """Runs that cross the 64 sequences of a planning wave and the 256 of a work-group's own plan."""
    rng = random.Random(batch)
    groups, left = [], batch
    while left:
        n = min(left, rng.choice((1, 2, 30, 70)))
        groups.append((rng.choice((4, 9, 44)) if n > 1 else 0, [rng.choice((None, 1, 20, 50)) if n < 30 else rng.randint(1, 50) for _ in range(n)]))
        left -= n
    b = Batch(groups, 16, 64, 2, 2, seed=batch, slots=True)
    b.both()


@pytest.mark.parametrize("d,kv,gq,q_len", [(64, 5, 1, 1), (96, 3, 4, 3), (128, 8, 5, 4), (64, 6, 20, 2)])
@pytest.mark.parametrize("longest", [100, 400, 2000])
def test_more_heads_than_groups(gpu_lib, d, kv, gq, q_len, longest):
    """So many sequences and heads that short tails are a wave's each, four heads a group; heads that 4 does not
    divide, tails on both sides of what a wave takes, whole tables that are never cut."""
    rng = random.Random(d + kv)
    tails = [rng.choice((None, 1, 2, q_len, 31, 32, 33, 64, 100, 127, 128, 129, 160)) for _ in range(600 // kv)]
    tails = [x if x is None else min(x, longest) for x in tails] + [longest]
    b = Batch([(0, tails[:40]), (3, tails[40:60]), (0, tails[60:])], 32, d, kv, gq, q_len, seed=longest)
    b.both()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("members", [2, 17, 40])
def test_shared_prefix(gpu_lib, page, d, members):
    """One group: 4 query heads a key-value head, so 8, 68 and 160 rows share the prefix."""
    rng = random.Random(members)
    b = Batch([(up(200, page), [rng.randint(1, 90) for _ in range(members)])], page, d, 2, 4, seed=page + d + members)
    b.both()


@pytest.mark.parametrize("gq,q_len", [(1, 2), (1, 128), (4, 5), (8, 4), (8, 16), (3, 11), (128, 1), (16, 2), (33, 1), (17, 3)])
@pytest.mark.parametrize("d,page", [(64, 16), (96, 64), (128, 32)])
def test_query_rows(gpu_lib, gq, q_len, d, page):
    """Several tokens a sequence and wide groups of heads; the first tokens of short sequences see nothing."""
    tails = [1, q_len, q_len + 1, max(1, q_len - 1), 70, 129, None, 40]
    b = Batch([(0, tails), (up(150, page), [q_len, q_len + 60, q_len + 7])], page, d, 1, gq, q_len, seed=gq * q_len, slots=True)
    b.both()


@pytest.mark.parametrize("d,page", [(64, 32), (96, 16), (128, 128)])
def test_drafts_longer_than_tails(gpu_lib, d, page):
    """Queries that reach back into the shared pages: these stay out of what is read once."""
    b = Batch([(4, [0, 1, 5, 0]), (2, [3, 0])], page, d, 2, 2, q_len=9, seed=5)
    b.both()


@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 64), (128, 128)])
def test_groups(gpu_lib, d, page):
    """Several prompts in a batch, single requests between, an empty slot, table rows in another order."""
    groups = [(3, [5, 60, 1]), (0, [40]), (7, [9] * 12), (0, [None]), (0, [None, 3]), (1, [33, 2]), (12, [100] * 33)]
    b = Batch(groups, page, d, 3, 2, seed=d + page, slots=True)
    b.both()


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("heads", [(1, 1), (5, 1), (2, 8)])
def test_long(gpu_lib, d, heads):
    """A long key axis split over many work-groups and joined, with and without sharing."""
    b = Batch([(500, [1, 777, 16]), (0, [9000])], 16, d, *heads, seed=d)
    b.both()


@pytest.mark.parametrize("d,page", [(64, 64), (128, 16)])
def test_many_sequences(gpu_lib, d, page):
    rng = random.Random(d)
    b = Batch([(2, [rng.randint(1, 60) for _ in range(300)]), (0, [rng.randint(1, 60) for _ in range(724)])], page, d, 1, 1, seed=d)
    b.both()


@pytest.mark.parametrize("gain,scale", [(60.0, 0.0), (1.0, 3.0), (0.0, 0.0), (1.0, 1e-6)])
def test_scores(gpu_lib, gain, scale):
    """Weights on one key, flat weights, a given scale."""
    b = Batch([(9, [40, 7, 3, 90] * 3), (0, [300])], 32, 128, 2, 4, seed=3, gain=gain)
    b.both(scale)


def test_scores_that_overflow(gpu_lib):
    """Keys of the largest finite values: scores past the fp32 range below give weight 0, not NaN."""
    b = Batch([(5, [20, 50, 33])], 16, 64, 1, 4, seed=8)
    big = torch.finfo(torch.bfloat16).max
    for s in b.ids:
        p = int(b.tables[s, int(b.lens[s] - 1) // 16])
        b.pool[0, p, :, 0] = -big
    b.q = b.q.abs() + 1
    b.cache.pool.copy_(b.pool)
    out, lse = b.run()
    keep = b.pool.clone()
    for s in b.ids:                                   # those keys hold no weight: the same without them
        p = int(b.tables[s, int(b.lens[s] - 1) // 16])
        b.pool[0, p, :, 0] = -1e4
    b.check(out, lse)
    b.pool = keep


@pytest.mark.parametrize("roomy", [False, True])
def test_infinite_keys_and_values(gpu_lib, roomy):
    """An infinite or NaN value makes the rows that see it non-finite in its dim, and no other row or dim."""
    b = Batch([(3, [30, 40, 50, 60])], 16, 64, 2, 2, q_len=3, seed=9)
    if roomy:
        b.cache = b.roomy()
    ref, _ = b.run()
    p = int(b.tables[b.ids[2], 5])                    # sequence 2's newest full page, private
    pos = int(b.lens[b.ids[2]]) - 1                   # its newest token: only the last query sees it
    p, at = int(b.tables[b.ids[2], pos // 16]), pos % 16
    for bad in (float("inf"), float("nan")):
        b.cache.pool.copy_(b.pool)
        b.cache.pool[1, p, 0, at, 7] = bad
        out, _ = b.run()
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[2, :2, 2, 7] = True                       # kv head 0, last token, dim 7
        assert not torch.isfinite(out[hit]).any()
        assert torch.equal(out[~hit], ref[~hit]), bad
        b.cache.pool.copy_(b.pool)
        b.cache.pool[0, p, 1, at, 3] = bad if bad != bad else -bad
        out, _ = b.run()
        rest = torch.ones_like(out, dtype=torch.bool)
        rest[2, 2:, 2] = False                        # kv head 1, last token
        assert torch.equal(out[rest], ref[rest]), bad


@pytest.mark.parametrize("members", [4, 40])
def test_nan_query(gpu_lib, members):
    """A NaN in one query makes that row NaN and changes no bit of the others."""
    b = Batch([(30, [5, 70, 200, 33] * (members // 4))], 16, 128, 2, 4, seed=16)
    refs = [b.run(shared)[0] for shared in (True, False)]
    b.q[1, 5, 0, 100] = float("nan")
    for shared, ref in zip((True, False), refs):
        out, lse = b.run(shared)
        rest = torch.ones(out.shape[:3], dtype=torch.bool, device="cuda")
        rest[1, 5, 0] = False
        assert torch.isnan(out[1, 5, 0]).all() and torch.isnan(lse[1, 5, 0])
        assert torch.equal(out[rest], ref[rest])


def test_bad_tables_and_lengths(gpu_lib):
    """Page ids outside the pool are not read, their positions not attended; lengths past the table and below 0 are cut."""
    b = Batch([(4, [30, 70, 20, 40]), (0, [100])], 16, 64, 1, 4, seed=4)
    ids = b.ids
    b.tables[ids[1], 5], b.tables[ids[3], 4] = b.pool.shape[1], -7
    b.tables[ids[2], 4] = 2 ** 31 - 1
    for s in ids[:4]:
        b.tables[s, 1] = -1                           # inside the shared pages
    cols = b.tables.shape[1]
    b.tables[ids[4], 3] = -2 ** 31
    b.lens[ids[0]] = -5
    b.cache.tables.copy_(ints(b.tables.tolist()))
    b.cache.lens.copy_(ints(b.lens.tolist()))
    b.both()
    full = [s for s in ids if b.tables[s, cols - 1] >= 0][0]
    b.pool.nan_to_num_(0.5)
    b.cache.pool.copy_(b.pool)
    b.lens[full] = cols * 16 + 1000
    b.cache.lens.copy_(ints(b.lens.tolist()))
    b.both()


def test_bad_page_shared_by_many(gpu_lib):
    """A missing page under more rows than a piece of few has: those positions stay out for all of them."""
    b = Batch([(40, [5, 9, 20] * 10)], 16, 64, 2, 4, seed=14)
    for s in b.ids:
        b.tables[s, 17] = -1
        b.tables[s, 39] = b.pool.shape[1] + 5
    b.cache.tables.copy_(ints(b.tables.tolist()))
    b.both()


@pytest.mark.parametrize("members", [3, 30])
def test_infinite_shared_value(gpu_lib, members):
    """An infinite value in a shared page reaches every row of its head, in its dim alone."""
    b = Batch([(40, [5, 9, 20] * (members // 3))], 16, 96, 2, 4, seed=15)
    ref, _ = b.run()
    b.cache.pool[1, int(b.tables[b.ids[0], 12]), 1, 3, 50] = float("inf")
    for shared in (True, False):
        out, _ = b.run(shared)
        assert not torch.isfinite(out[:, 4:, :, 50]).any()
        keep = [i for i in range(96) if i != 50]
        assert torch.isfinite(out[..., keep]).all() and torch.isfinite(out[:, :4]).all()
        if shared:
            assert torch.equal(out[..., keep], ref[..., keep]) and torch.equal(out[:, :4], ref[:, :4])


def reference_on_gpu(q, k, v):
    """(o, lse, bound, lse_bound) as cache_model.attend gives them, of rows q [rows][d] that see every key, by torch in fp64."""
    d = q.shape[-1]
    scale = float(np.float32(1 / np.sqrt(d)))
    q, k, v = q.double(), k.double(), v.double()
    x = (q @ k.t()) * scale
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    o = p @ v
    e = scale * d * 2.0 ** -24 * (q.abs() @ k.abs().t()).amax(1, keepdim=True)
    bound = 2.0 ** -8 * o.abs() + (1 + 2.0 ** -8) * (2.0 ** -8 + 2 * e + 2.0 ** -16) * (p @ v.abs())
    return o, lse, bound, e[:, 0] + 2.0 ** -16 + 2.0 ** -22 * lse.abs()


@pytest.mark.parametrize("batch,kv,gq,page,tokens", [(1, 16, 2, 128, 300001), (128, 8, 4, 64, 40000), (20, 8, 4, 16, 120000)])
def test_pieces_of_more_than_4096_keys(gpu_lib, batch, kv, gq, page, tokens):
    """So many keys that a piece is longer than the page ids that a wave holds at once, for one sequence and shared."""
    d = 64
    say(f"{batch} sequences over {tokens} tokens, {kv} heads")
    g = torch.Generator(device="cuda").manual_seed(batch)
    cols = up(tokens, page)
    n = tokens // page * page                         # shared by all; each has up to a page of its own
    pool = torch.randn((2, cols + batch, kv, page, d), generator=g, device="cuda").to(torch.bfloat16)
    order = torch.randperm(cols + batch, generator=g, device="cuda").to(torch.int32)
    tables = order[:cols][None].repeat(batch, 1)
    tables[:, n // page:] = order[cols:cols + batch, None]
    tables = tables[:, :up(tokens, page)].contiguous()
    lens = torch.full((batch,), tokens, dtype=torch.int32, device="cuda")
    c = PagedCache(1, cols + batch, page, kv, d, batch, tables.shape[1], pool=pool, tables=tables, lens=lens)
    q = torch.randn((batch, kv * gq, 1, d), generator=g, device="cuda").to(torch.bfloat16)
    shared = torch.full((batch,), n // page, dtype=torch.int32, device="cuda")
    shared[0] = 0
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    c.attend(0, q, out, lse, shared=shared if batch > 1 else None)
    for b in (0, batch - 1):
        for h in (0, kv - 1):
            k, v = (pool[x, tables[b].long(), h].reshape(-1, d)[:tokens] for x in (0, 1))
            rows = slice(h * gq, (h + 1) * gq)
            o, z, bound, zb = reference_on_gpu(q[b, rows, 0], k, v)
            assert ((out[b, rows, 0].double() - o).abs() <= bound).all()
            assert ((lse[b, rows, 0].double() - z).abs() <= zb).all()


def test_repeated_and_foreign_ids(gpu_lib):
    b = Batch([(2, [30, 5]), (0, [9])], 16, 64, 2, 2, seed=6)
    b.ids = [b.ids[0], b.ids[0], b.ids[2]]
    b.shared = [0, 4, -3]
    b.both()
    b.ids = [99, b.ids[0], -1]
    b.shared = [5, 2, 2]
    b.both()


def test_shared_larger_than_it_is(gpu_lib):
    """shared is cut to what every member of a run holds."""
    b = Batch([(2, [30, 5, 1])], 16, 64, 2, 2, seed=7)
    b.shared = [77, 2, 10 ** 9]
    b.both()


def test_rows_are_left_alone(gpu_lib):
    """Nothing is written behind the batch's rows."""
    b = Batch([(2, [30, 5, 1] * 5)], 16, 96, 2, 2, seed=7)
    big = torch.full((b.q.numel() + 4096,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[:b.q.numel()].view(b.q.shape)
    b.check(*b.run(out=out))
    assert bool((big[b.q.numel():] == 7).all())


def test_long_pool(gpu_lib):
    """Pages past 4 GB of a plane."""
    d, kv, page = 128, 8, 128
    pages = 20000                                     # 5.2 GB a plane
    c = PagedCache(1, pages, page, kv, d, 2, 3, pool=torch.empty((2, pages, kv, page, d), dtype=torch.bfloat16, device="cuda"))
    c.tables.copy_(ints([[19999, 3, 17001], [19999, 18888, -1]]))
    c.lens.copy_(ints([300, 200]))
    g = torch.Generator(device="cuda").manual_seed(1)
    used = [19999, 3, 17001, 18888]
    small = torch.randn((2, 4, kv, page, d), generator=g, device="cuda").to(torch.bfloat16)
    c.pool[:, used] = small
    q = torch.randn((2, 2 * kv, 1, d), generator=g, device="cuda").to(torch.bfloat16)
    want = PagedCache(1, 4, page, kv, d, 2, 3, pool=small, tables=ints([[0, 1, 2], [0, 3, -1]]), lens=ints([300, 200]))
    outs = []
    for x in (c, want):
        for sh in (None, ints([0, 1])):
            outs.append(x.attend(0, q, torch.empty_like(q), shared=sh))
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
    # moves of such pages: the copy of a shared last page, and compaction
    c.refs.zero_()
    c.refs[ints(used).long()] = ints([2, 1, 1, 1])
    live = c.compact()
    torch.cuda.synchronize()
    assert int(live) == 4
    # 3 stays; the others go to 0, 1, 2 in ascending order
    assert c.tables.cpu().tolist() == [[2, 3, 0], [2, 1, -1]]
    assert torch.equal(c.pool[:, [2, 3, 0, 1]], small)


def test_long_pool_many_rows(gpu_lib):
    """The same for what many rows share, and for what reserve, append and its copies write there."""
    d, kv, page, pages, n = 128, 8, 128, 20000, 24
    c = PagedCache(1, pages, page, kv, d, n, 20, pool=torch.empty((2, pages, kv, page, d), dtype=torch.bfloat16, device="cuda"))
    small = PagedCache(1, 64, page, kv, d, n, 20)
    c.refs.fill_(1)
    c.refs[-64:] = 0                                  # only the last pages are free
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((1, kv, 1000, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    k2, v2 = (torch.randn((n, kv, 2, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((n, 4 * kv, 1, d), generator=g, device="cuda").to(torch.bfloat16)
    ids, outs = ints(list(range(n))), []
    for x in (c, small):
        x.append(0, k, v, ints([0]), x.reserve(ints([0]), ints([1000])))
        assert x.fork(ints([0] * (n - 1)), ints(list(range(1, n)))).sum() == n - 1
        x.append(0, k2, v2, ids, x.reserve(ids, ints([2] * n)))   # 24 copies of the last page
        outs.append(x.attend(0, q, torch.empty_like(q), shared=x.shared()))
    used = small.tables >= 0
    assert used.sum() == 8 * n and torch.equal(c.tables[used], small.tables[used] + pages - 64)
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1])
    assert torch.equal(small.shared().cpu(), torch.tensor([0] + [7] * (n - 1), dtype=torch.int32))


def test_two_graphs_of_one_cache(gpu_lib):
    """Two captured calls of one shape use one workspace, in turn."""
    b = Batch([(50, [30, 5, 64, 100] * 6), (0, [900])], 16, 64, 2, 4, seed=17)
    sh, ids = ints(b.shared), ints(b.ids)
    qs = [b.q.cuda(), b.q.flip(0).cuda()]
    eager = [b.cache.attend(0, q, torch.empty_like(q), seq_ids=ids, shared=s).clone() for q, s in zip(qs, (sh, None))]
    outs, graphs = [torch.empty_like(q) for q in qs], []
    for q, o, s in zip(qs, outs, (sh, None)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            b.cache.attend(0, q, o, seq_ids=ids, shared=s)
    for rep in range(3):
        for o in outs:
            o.fill_(float("nan"))
        for i in (0, 1) if rep % 2 else (1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, e) for o, e in zip(outs, eager))
        b.cache.attend(0, qs[0], torch.empty_like(qs[0]), seq_ids=ids, shared=sh)


def test_graph_and_streams(gpu_lib):
    """Replays of a captured call between eager ones, with lengths changing; calls of two shapes on two streams."""
    b = Batch([(5, [30, 5, 64, 100] * 9), (0, [200])], 16, 128, 2, 4, seed=11)
    q, sh, ids = b.q.cuda(), ints(b.shared), ints(b.ids)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    eager = [t.clone() for t in b.run()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.cache.attend(0, q, out, lse, seq_ids=ids, shared=sh)
    full = b.cache.lens.clone()
    for rep in range(4):
        b.cache.lens.copy_(full - 4 * (rep % 2))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = b.run()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        if rep % 2 == 0:
            assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
    other = Batch([(0, [900, 30])], 64, 64, 3, 1, seed=12)
    first, second = b.run()[0].clone(), other.run()[0].clone()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    o1, o2, q2 = torch.empty_like(q), torch.empty_like(second), other.q.cuda()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            b.cache.attend(0, q, o1, seq_ids=ids, shared=sh)
        with torch.cuda.stream(s2):
            other.cache.attend(0, q2, o2)
    torch.cuda.synchronize()
    assert torch.equal(o1, first) and torch.equal(o2, second)


def test_after_a_prompt(gpu_lib):
    """A prompt's keys and values go into the cache and its last token attends: the dense call's last row."""
    w = gpu_lib
    n, heads, kv, d = 320, 8, 2, 96
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((2, h, n, d), generator=g, device="cuda").to(torch.bfloat16) for h in (heads, kv, kv))
    o, lse = torch.empty_like(q), torch.empty((2, heads, n), dtype=torch.float32, device="cuda")
    w.wise_dense_attn_accum(w.make_shape(2, heads, n, d, 64, kv_heads=kv), q, k, v, o, lse)
    c = PagedCache(1, 30, 32, kv, d, 4, 12)
    ids = ints([2, 0])
    c.append(0, k, v, ids, c.reserve(ids, ints([n, n])))
    last, z = torch.empty((2, heads, 3, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, heads, 3), device="cuda")
    c.attend(0, q[:, :, -3:].contiguous(), last, z, seq_ids=ids)
    torch.cuda.synchronize()
    # Both are within 2^-8 |o| + 2^-8 A (rounded output, rounded probabilities) of the definition; |v| < 6 gives A < 6.
    assert (last.float() - o[:, :, -3:].float()).abs().max() <= 2 * (2 ** -8 * 6 + 2 ** -8 * 6)
    assert (z - lse[:, :, -3:]).abs().max() <= 1e-4


@pytest.mark.parametrize("name,groups,kv,gq,q_len,cut", [
    ("a row a sequence, whole", [(0, [1, 40, 300, 512])], 2, 4, 1, False),
    ("a row a sequence, cut", [(0, [700, 1500, 33])], 2, 4, 1, True),
    ("two row tiles", [(0, [700, 90])], 1, 6, 4, True),
    ("a wave alone", [(0, [20, 64, 100, 128] * 40)], 4, 1, 1, True),
    ("few rows share", [(12, [9, 40, 130])], 2, 4, 1, True),
    ("many rows share", [(24, [9, 40, 130] * 8)], 2, 4, 1, True)])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_probabilities_keep_their_bits(gpu_lib, name, groups, kv, gq, q_len, cut, d):
    """The probabilities enter the product with 16 bits: half a step of bf16 is left of each by the first part, and half
    a step of that by the second, 2^-16 instead of the 2^-8 of the general bound."""
    b = Batch(groups, 32, d, kv, gq, q_len, seed=d)
    f64 = lambda t: bf16_values(t.view(torch.int16).numpy())  # noqa: E731
    q, k, v = f64(b.q), f64(b.pool[0]), f64(b.pool[1])
    scale = float(np.float32(1 / np.sqrt(d)))
    o, _, bound, _ = attend(q, k, v, b.tables, b.lens, b.ids, b.page, scale)
    rest = (bound - 2.0 ** -8 * np.abs(o)) / (1 + 2.0 ** -8)          # (2^-8 + 2 e + 2^-16) A
    weight = attend(q, k, np.abs(v), b.tables, b.lens, b.ids, b.page, scale)[0]
    bound = 2.0 ** -8 * np.abs(o) + (1 + 2.0 ** -8) * (rest + (2.0 ** -16 - 2.0 ** -8) * weight)
    for shared in (True, False):
        out, _ = b.run(shared, cache=b.roomy() if cut else None)
        err = np.abs(out.double().cpu().numpy() - o)
        assert np.all(err <= bound), f"{name}: {np.max(err / bound):.3g} of the bound"


def own_pages_gone(b, runs):
    """b's cache in roomy tables where a run's sequences but its first name a page of NaN in place of the pages that the
    run shares: only a call that reads these through the first one's table gives numbers.  runs: (first, end, pages)."""
    cache = b.roomy()
    nan = int(torch.isnan(b.pool).all(dim=4).all(dim=3).all(dim=2).all(dim=0).nonzero()[0])
    for first, end, pages in runs:
        for i in range(first + 1, end):
            cache.tables[b.ids[i], :pages] = nan
    return cache


@pytest.mark.parametrize("border", [1, 4, 5, 20])
@pytest.mark.parametrize("groups", [[(40, 8), (30, 9)], [(40, 20), (0, 1), (40, 33)], [(100, 30), (60, 30), (21, 30), (77, 30)],
                                    [(30, 100)] * 3])
def test_runs_that_share_little(gpu_lib, groups, border):
    """Families of requests with a few common pages, or a single request among them: each family's pages are still read once."""
    rng = random.Random(border)
    b = Batch([(pre, [rng.randint(1, 40) for _ in range(n)]) for pre, n in groups], 32, 64, 32, 1, seed=border, slots=True)
    runs, at = [], 0
    for pre, n in groups:
        runs.append((at, at + n, pre // 2 * 2))
        at += n
    want, _ = b.run(cache=b.roomy())
    for first, _, _ in runs[1:]:
        b.shared[first] = border                      # of the pages of this family and the one before
    out, _ = b.run(cache=own_pages_gone(b, runs))
    assert torch.isfinite(want).all() and torch.equal(out, want)


def test_one_short_request_in_a_run(gpu_lib):
    """A sequence of a few tokens in the middle of users of a long prompt, as shared() counts it."""
    b = Batch([(64, [9, 30, 5] * 10), (0, [70]), (64, [9, 30, 5] * 11)], 64, 64, 2, 4, seed=19)
    for i in range(30, 64):                           # the same first page and, but for the short one, the same prompt
        n = 1 if i == 30 else 64
        b.tables[b.ids[i], :n] = b.tables[b.ids[0], :n]
    b.cache.tables.copy_(ints(b.tables.tolist()))
    b.shared = b.cache.shared(ints(b.ids)).cpu().tolist()
    assert b.shared == [0] + [64] * 29 + [1, 1] + [64] * 32
    cache = b.roomy()
    b.check(*b.run(cache=cache))
    out, _ = b.run(cache=own_pages_gone(b, [(0, 30, 64), (31, 64, 64)]))
    assert torch.equal(out, b.run(cache=cache)[0])


@pytest.mark.parametrize("threads,samples,system,thread", [(8, 8, 32, 20), (3, 40, 40, 20), (40, 3, 16, 64), (2, 3, 16, 240)])
def test_samples_of_threads(gpu_lib, threads, samples, system, thread):
    """Samples of several threads under one system prompt: what a thread's samples share is read once for each thread where
    that saves more than the system prompt read once for all."""
    b = Batch([(system + thread, [1, 30, 7, 12][:samples] * (samples // min(samples, 4)))] * threads, 64, 64, 4, 1, seed=threads)
    n = len(b.ids) // threads
    for i in range(n, len(b.ids)):
        b.tables[b.ids[i], :system] = b.tables[b.ids[0], :system]
    b.cache.tables.copy_(ints(b.tables.tolist()))
    b.shared = b.cache.shared(ints(b.ids)).cpu().tolist()
    assert b.shared == ([0] + ([system + thread] * (n - 1) + [system]) * threads)[:len(b.ids)]
    assert threads * (n - 1) * (system + thread) > (len(b.ids) - 1) * system
    cache = b.roomy()
    want, lse = b.run(cache=cache)
    b.check(want, lse)
    out, _ = b.run(cache=own_pages_gone(b, [(i * n, i * n + n, system + thread) for i in range(threads)]))
    assert torch.equal(out, want)


def test_a_little_more_is_not_worth_a_cut(gpu_lib):
    """Pairs that share a page more than all do stay in one run, which reads what all share once."""
    b = Batch([(40, [280, 290, 300, 270] * 9)], 64, 64, 32, 1, seed=20)
    b.shared = [0] + [40 + 4 * (i % 2) for i in range(1, 36)]
    for i in range(2, 36, 2):                         # 44 pages of sequence i are those of i - 1
        b.shared[i] = 40
    for i in range(1, 36, 2):
        b.tables[b.ids[i], 40:44] = b.tables[b.ids[i - 1], 40:44]
    b.cache.tables.copy_(ints(b.tables.tolist()))
    cache = b.roomy()
    want, lse = b.run(cache=cache)
    b.check(want, lse)
    assert torch.equal(b.run(cache=own_pages_gone(b, [(0, 36, 40)]))[0], want)


class Uneven(Batch):
    """Sequences that each share some leading pages with the one before, of any number."""

    def __init__(self, batch, page, d, kv, gq, q_len, most, seed):
        super().__init__([(0, [1])], page, d, kv, gq, q_len, seed=seed)
        rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
        rows, lens, at = [], [], 0
        for i in range(batch):
            k = rng.choice((0, 1, rng.randint(0, most), most)) if rows else 0
            row = rows[-1][:min(k, lens[-1] // page)] if rows else []
            n = len(row) * page + rng.choice((0, 1, rng.randint(0, 2 * page), rng.randint(0, most * page - len(row) * page)))
            new = up(n, page) - len(row)
            rows.append(row + list(range(at, at + new)))
            lens.append(n)
            at += new
        cols = max(1, max(map(len, rows)), 2048 // page + 2)
        self.tables, self.lens, self.ids = np.full((batch, cols), -1), np.array(lens), list(range(batch))
        for i, row in enumerate(rows):
            self.tables[i, :len(row)] = row
        self.pool = torch.randn((2, at + 1, kv, page, d), generator=g).to(torch.bfloat16)
        self.q = torch.randn((batch, kv * gq, q_len, d), generator=g).to(torch.bfloat16)
        self.cache = PagedCache(1, at + 1, page, kv, d, batch, cols, pool=self.pool.cuda(), tables=ints(self.tables.tolist()), lens=ints(lens))
        self.shared = self.cache.shared().cpu().tolist()


@pytest.mark.parametrize("batch,q_len,most", [(2, 1, 512), (17, 3, 4096), (64, 1, 2048), (65, 2, 4096), (256, 1, 1024), (257, 2, 1024), (600, 1, 640)])
@pytest.mark.parametrize("page", [16, 64])
def test_uneven_sharing(gpu_lib, batch, q_len, most, page):
    """Any pattern of shared pages, as shared() gives it: the definition, and the same bits at every call."""
    for seed in range(2):
        b = Uneven(batch, page, 64, 8, 1, q_len, most // page, seed)
        out, lse = b.run()
        b.check(out, lse)
        again, lse2 = b.run()
        assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_one_workspace_for_all_shapes(gpu_lib):
    """A cache holds no more workspace than the largest of its calls needs (for the next power of two of its batch)."""
    w = gpu_lib
    c = PagedCache(1, 64, 64, 8, 128, 64, 128)
    shapes = [(b, q_len) for q_len in (1, 2, 3, 4, 5) for b in (1, 3, 17, 40, 64, 20)]
    need = max(w.wise_prefix_workspace_bytes(c.shape, w.make_queries(1 << (b - 1).bit_length(), 32, q_len)) for b, q_len in shapes)
    q = torch.zeros((64, 32, 5, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for b, q_len in shapes:
        c.attend(0, q[:b, :, :q_len].contiguous(), out.flatten()[:b * 32 * q_len * 128].view(b, 32, q_len, 128))
    torch.cuda.synchronize()
    assert need <= torch.cuda.memory_allocated() - before <= need + (4 << 20)


@pytest.mark.parametrize("eager_first", [False, True])
def test_a_graph_keeps_its_workspace(gpu_lib, eager_first):
    """A larger eager call after a capture, and other tensors in whatever memory it freed: replays use what they captured."""
    b = Batch([(50, [30, 5, 64, 100]), (0, [900])], 16, 64, 2, 4, seed=21)
    big = torch.zeros((5, 8, 16, 64), dtype=torch.bfloat16, device="cuda")
    q, sh, ids = b.q.cuda(), ints(b.shared), ints(b.ids)
    eager, z = (t.clone() for t in b.run(cache=Batch([(50, [30, 5, 64, 100]), (0, [900])], 16, 64, 2, 4, seed=21).cache))
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    if eager_first:
        b.cache.attend(0, q, out, lse, seq_ids=ids, shared=sh)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.cache.attend(0, q, out, lse, seq_ids=ids, shared=sh)
    for rep in range(3):
        if rep == 1:
            b.cache.attend(0, big, torch.empty_like(big), seq_ids=ids)      # grows
        others = [torch.full((1 << 18,), float("nan"), device="cuda") for _ in range(64)]
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse, z)
        assert all(torch.isnan(t).all() for t in others)
    again = torch.cuda.CUDAGraph()                                          # one that grows it while it captures
    big2 = torch.zeros((5, 8, 32, 64), dtype=torch.bfloat16, device="cuda")
    out2 = torch.empty_like(big2)
    with torch.cuda.graph(again):
        b.cache.attend(0, big2, out2, seq_ids=ids, shared=sh)
    want2 = b.cache.attend(0, big2, torch.empty_like(big2), seq_ids=ids, shared=sh)
    for rep in range(2):
        out.fill_(float("nan"))
        out2.fill_(float("nan"))
        again.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(out2, want2)


def test_a_workspace_outgrown_on_another_stream(gpu_lib):
    """Calls in order on two streams, the second of which outgrows the workspace: its memory goes to nobody before the first is done."""
    b = Batch([(200, [30, 5, 64, 100] * 8)], 16, 64, 8, 4, seed=22)
    q, ids = b.q.cuda(), ints(b.ids)
    big = torch.zeros((32, 32, 8, 64), dtype=torch.bfloat16, device="cuda")
    want = b.run(shared=False)[0].clone()
    for rep in range(3):
        c = PagedCache(1, b.cache.shape.pages, 16, 8, 64, b.cache.shape.seqs, b.cache.shape.max_pages, pool=b.cache.pool, tables=b.cache.tables,
                       lens=b.cache.lens)
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        outs, out2 = [torch.empty_like(q) for _ in range(20)], torch.empty_like(big)
        torch.cuda.synchronize()
        with torch.cuda.stream(s1):
            for o in outs:
                c.attend(0, q, o, seq_ids=ids)
        s2.wait_stream(s1)
        with torch.cuda.stream(s2):
            c.attend(0, big, out2, seq_ids=ids)
        with torch.cuda.stream(s1):
            torch.full((1 << 24,), float("nan"), device="cuda")
        torch.full((1 << 24,), float("nan"), device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("d,kv,gq,batch", [(128, 8, 1, 150), (64, 8, 2, 300), (96, 16, 1, 100), (64, 1, 8, 1024)])
def test_many_sequences_of_short_tables(gpu_lib, d, kv, gq, batch):
    """Tables of 512 tokens whose K and V, all read for themselves, would be more than 256 MB: what they share is read once."""
    b = Batch([(14, [1 + 5 * i % 64 for i in range(batch)])], 32, d, kv, gq, seed=d + kv)
    assert b.cache.shape.max_pages * 32 == 512
    b.check(*b.run())
    b.check(*b.run(shared=False))
    if batch * kv * 512 * d * 4 > 256 << 20:
        want = b.run()[0].clone()
        nan = int(torch.isnan(b.pool).all(dim=4).all(dim=3).all(dim=2).all(dim=0).nonzero()[0])
        b.cache.tables[1:batch, :14] = nan
        assert torch.isfinite(want).all() and torch.equal(b.run()[0], want)


def test_after_a_prompt_element_by_element(gpu_lib):
    """The prompt's K and V go into the cache by append, and its last tokens attend as in the dense call: both are held, element by
    element, to the definition computed from the prompt itself, closely enough that one value in the wrong place shows."""
    w = gpu_lib
    n, heads, kv, d, q_len = 320, 8, 2, 96, 3
    g = torch.Generator(device="cuda").manual_seed(23)
    q, k, v = (torch.randn((2, h, n, d), generator=g, device="cuda").to(torch.bfloat16) for h in (heads, kv, kv))
    dense = torch.empty_like(q)
    w.wise_dense_attn_accum(w.make_shape(2, heads, n, d, 64, kv_heads=kv), q, k, v, dense)
    c = PagedCache(1, 30, 32, kv, d, 4, 12)
    ids = ints([2, 0])
    c.append(0, k, v, ids, c.reserve(ids, ints([n, n])))
    out, lse = torch.empty((2, heads, q_len, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, heads, q_len), device="cuda")
    c.attend(0, q[:, :, -q_len:].contiguous(), out, lse, seq_ids=ids)
    gq, seen = heads // kv, set()
    for b in range(2):
        for h in range(heads):
            for t in range(q_len):
                see = n - q_len + 1 + t
                row, keys, values = q[b, h, see - 1][None], k[b, h // gq, :see], v[b, h // gq, :see]
                o, z, bound, zb = reference_on_gpu(row, keys, values)
                # the cache's probabilities have 16 bits in the product, the dense kernel's 8
                weight = reference_on_gpu(row, keys, values.abs())[0]
                close = bound + (1 + 2.0 ** -8) * (2.0 ** -16 - 2.0 ** -8) * weight
                assert ((out[b, h, t].double() - o[0]).abs() <= close[0]).all()
                assert ((lse[b, h, t].double() - z[0]).abs() <= zb[0])
                assert ((dense[b, h, see - 1].double() - o[0]).abs() <= bound[0]).all()
                # the newest token's values missing, or those of two tokens exchanged, would be seen
                for i, wrong in enumerate((torch.cat([values[:-1], torch.zeros_like(values[:1])]), values[[1, 0] + list(range(2, see))])):
                    off = reference_on_gpu(row, keys, wrong)[0]
                    if ((out[b, h, t].double() - off[0]).abs() > close[0]).any():
                        seen.add((i, b, h // gq))
    assert len(seen) == 2 * 2 * kv                    # by some row of every key-value head


@pytest.mark.parametrize("name,groups,kv,gq,q_len,cut", [
    ("a row a sequence, whole", [(4, [40, 300, 200])], 2, 4, 1, False),
    ("a row a sequence, cut", [(4, [700, 1500, 33])], 2, 4, 1, True),
    ("two row tiles", [(4, [700, 90])], 1, 6, 4, True),
    ("a wave alone", [(2, [20, 40, 61] * 54)], 4, 1, 1, True),
    ("few rows share", [(12, [9, 40, 130])], 2, 4, 1, True),
    ("many rows share", [(24, [9, 40, 130] * 8)], 2, 4, 1, True)])
@pytest.mark.parametrize("scale", [0.0, 40.0])
@pytest.mark.parametrize("at", [3, 60])
def test_infinite_values_that_are_seen(gpu_lib, name, groups, kv, gq, q_len, cut, scale, at):
    """A row that sees an infinite value gets it, whatever its weight (at a scale of 40 most vanish); NaN where it sees one, or
    both infinities; the other dims are as they were."""
    b = Batch(groups, 32, 96, kv, gq, q_len, seed=24)
    page = int(b.tables[b.ids[0], at // 32])          # of the shared ones
    cache = b.roomy() if cut else b.cache
    inf = float("inf")
    for shared in (True, False):
        cache.pool.copy_(b.pool)
        ref, zref = (t.clone() for t in b.run(shared, scale, cache=cache))
        v = cache.pool[1, page, kv - 1]
        v[at % 32, 7], v[at % 32, 95], v[at % 32, 40], v[at % 32 + 1, 64], v[at % 32 + 3, 64] = inf, -inf, float("nan"), inf, -inf
        out, lse = b.run(shared, scale, cache=cache)
        hit = out[:, (kv - 1) * gq:].float()
        assert (hit[..., 7] == inf).all() and (hit[..., 95] == -inf).all()
        assert torch.isnan(hit[..., 40]).all() and torch.isnan(hit[..., 64]).all()
        keep = [i for i in range(96) if i not in (7, 95, 40, 64)]
        assert torch.equal(out[..., keep], ref[..., keep]) and torch.equal(out[:, :(kv - 1) * gq], ref[:, :(kv - 1) * gq])
        assert torch.equal(lse, zref)
