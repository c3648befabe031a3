"""Performance cases of the paged key-value cache and of the attention that reads it.

A program that generates after a prompt keeps its keys and values in pages of
a pool ([layers x {K, V}][pages][kv_heads][page][head_dim], bf16), with a page
table, a length and the pages' reference counts on the device.  A case is one
of the things that it does with them, through `PagedCache`:

  attn     attention of a batch's newest tokens over their pages; sequences
           that share a prompt name the same pages, which are read once for all
  step     what comes before it: sequences dropped back to their accepted
           length, forks, room for the new tokens (a shared last page is
           copied), the tokens' keys and values into every layer, and which
           neighbours of the batch share their pages
  compact  requests admitted and finished, then the live pages moved to the
           front of the pool

With `own` false the same is computed in elementary torch operations.
"""

import math
import random

import torch

own = False


def _attn(batch, heads, kv_heads, d, page, q_len, groups, prefix, tail_min, tail_max, slots=False, mix=0):
    return dict(kind="attn", batch=batch, heads=heads, kv_heads=kv_heads, d=d, page=page, q_len=q_len, groups=groups, prefix=prefix,
                tail_min=tail_min, tail_max=tail_max, slots=slots, mix=mix)


def _step(layers, kv_heads, d, page, parents, children, len_min, len_max, tokens_min, tokens_max, mix=0):
    return dict(kind="step", layers=layers, kv_heads=kv_heads, d=d, page=page, parents=parents, children=children, len_min=len_min, len_max=len_max,
                tokens_min=tokens_min, tokens_max=tokens_max, mix=mix)


def _compact(layers, kv_heads, d, page, base, admitted, len_min, len_max, finished, mix=0):
    return dict(kind="compact", layers=layers, kv_heads=kv_heads, d=d, page=page, base=base, admitted=admitted, len_min=len_min, len_max=len_max,
                finished=finished, mix=mix)


def listed():
    cases = {
        # One user's next token, a short text, grouped-query heads of 64: the call's latency.
        "attn_one_short": _attn(1, 32, 8, 64, 32, 1, 1, 0, 301, 301),
        # A serving batch of unrelated requests, 4K tokens at most, grouped-query heads of 128: plain paged attention.
        "attn_ragged_4k": _attn(32, 32, 8, 128, 64, 1, 1, 0, 1, 4096, mix=1),
        # Eight samples of one 4K prompt at the paper's geometry (55 heads of 96, 32-key blocks), up to 256 tokens each.
        "attn_samples_4k": _attn(8, 55, 55, 96, 32, 1, 1, 4096, 1, 256, mix=2),
        # A system prompt of 8K tokens under 64 users' own turns.
        "attn_system_8k": _attn(64, 32, 8, 128, 64, 1, 1, 8192, 1, 1024, mix=3),
        # Six tasks with few-shot prompts of their own, 47 requests, the finest pages, table rows in the scheduler's order.
        "attn_tasks": _attn(47, 32, 8, 64, 16, 1, 6, 2032, 1, 333, slots=True, mix=4),
        # Five drafted tokens a sequence checked at once, 16 samples of a 4K prompt.
        "attn_drafts_4k": _attn(16, 32, 8, 128, 128, 5, 1, 4096, 5, 700, mix=5),
        # The largest: a 32K document and 128 users' questions about it with their answers.
        "attn_document_32k": _attn(128, 32, 8, 128, 128, 1, 1, 32768, 1, 4096, mix=6),
        # One prompt of a small model forked into four samples, one token each: launches count.
        "step_fork_small": _step(1, 8, 64, 16, 1, 4, 100, 100, 1, 1),
        # A wide sampling step: 16 prompts of 8 samples at the paper's geometry (4 layers x 55 heads of 96), 128 last pages copied.
        "step_samples": _step(4, 55, 96, 32, 16, 8, 500, 1500, 1, 1, mix=7),
        # Prompts of up to 4K tokens entering the cache of a 6-layer grouped-query model.
        "step_prompts_4k": _step(6, 8, 64, 64, 8, 0, 0, 0, 700, 4096, mix=8),
        # A small pool after a few short requests have finished.
        "compact_small": _compact(1, 8, 64, 16, 3, 12, 20, 200, 5, mix=9),
        # A serving pool of 4 layers after half of 64 requests of up to 4K tokens have finished.
        "compact_4k": _compact(4, 8, 128, 64, 16, 64, 500, 4096, 32, mix=10),
    }
    return [dict(c, name=k) for k, c in cases.items()]


def draw(rng):
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("attn", "attn", "attn", "step", "compact"))
    d, page, mix = rng.choice((64, 96, 128)), rng.choice((16, 32, 64, 128)), rng.randrange(1 << 20)
    gq = rng.choice((1, 2, 4, 8))
    kv = between(1, 55 if gq == 1 else 16)
    if kind == "attn":
        batch = between(1, 128)
        groups = min(batch, rng.choice((1, 1, 1, 2, 3, 7)))
        prefix = page * (between(1, 32768 // page) if rng.random() < 0.7 else 0)
        q_len = rng.choice((1, 1, 1, rng.randint(2, 8)))
        tail = max(q_len, between(1, 4096))
        c = _attn(batch, kv * gq, kv, d, page, q_len, groups, prefix, max(q_len, tail // rng.choice((1, 2, 16, 1000))), tail, rng.random() < 0.3, mix)
        big = work(listed()[6])
        while work(c)["bytes"] > big["bytes"] or work(c)["flops"] > big["flops"]:
            c["batch"] = max(1, c["batch"] // 2)
            c["groups"] = min(c["groups"], c["batch"])
            c["tail_min"], c["tail_max"] = max(q_len, c["tail_min"] // 2), max(q_len, c["tail_max"] // 2)
        return c
    layers = rng.choice((1, 1, 2, 4, 6))
    if kind == "step":
        if rng.random() < 0.3:
            parents, children, hi, tok = between(1, 16), 0, between(1, 512), between(1, 4096)
        else:
            parents, children, hi, tok = between(1, 24), between(1, 8), between(1, 2048), rng.choice((1, 1, rng.randint(2, 8)))
        c = _step(layers, kv, d, page, parents, children, max(1, hi // rng.choice((1, 3, 100))), hi, max(1, tok // rng.choice((1, 4))), tok, mix)
    else:
        n, hi = between(2, 64), between(page, 4096)
        c = _compact(layers, kv, d, page, rng.randint(0, 16), n, max(1, hi // rng.choice((1, 8))), hi, rng.randint(1, n - 1), mix)
    while _pool_bytes(c) > 2 << 30:                   # as much as the largest listed pool
        if c["layers"] > 1:
            c["layers"] -= 1
        else:
            c["len_max"] = max(1, c["len_max"] // 2)
            c["len_min"] = min(c["len_min"], c["len_max"])
            if kind == "step":
                c["tokens_max"] = max(1, c["tokens_max"] // 2)
                c["tokens_min"] = min(c["tokens_min"], c["tokens_max"])
    return c


# ---------------------------------------------------------------- the layout that a case means

def _up(x, y):
    return -(-x // y)


def _lengths(rng, n, lo, hi):
    """n lengths, one of them the longest."""
    out = [rng.randint(lo, hi) for _ in range(n)]
    if n:
        out[rng.randrange(n)] = hi
    return out


def _attn_layout(c):
    """Tables and lengths of the batch's sequences, the ids of their table rows, and the pages of the pool."""
    rng = random.Random(c["mix"])
    page, batch = c["page"], c["batch"]
    tails = _lengths(rng, batch, c["tail_min"], c["tail_max"])
    cuts = [0] + sorted(rng.sample(range(1, batch), c["groups"] - 1)) + [batch]
    head = [b in cuts for b in range(batch)]
    pre = c["prefix"] // page
    need = sum(_up(t, page) for t in tails) + pre * c["groups"]
    pages = need + need // 8 + 1
    free = list(range(pages))
    rng.shuffle(free)                                 # a pool that has been in use
    rows, lens, shared, first = [], [], [], []
    for b in range(batch):
        if head[b]:
            first = [free.pop() for _ in range(pre)]
        rows.append(first + [free.pop() for _ in range(_up(tails[b], page))])
        lens.append(c["prefix"] + tails[b])
        shared.append(0 if head[b] else pre)
    ids = list(range(batch))
    if c["slots"]:
        ids = rng.sample(range(batch + 3), batch)
    return rows, lens, shared, ids, pages, cuts


def _step_layout(c):
    """Parents' lengths, (source, destination) of the forks, the sequences that grow and by how much."""
    rng = random.Random(c["mix"])
    lens = _lengths(rng, c["parents"], c["len_min"], c["len_max"]) if c["len_max"] else [0] * c["parents"]
    src = [p for p in range(c["parents"]) for _ in range(c["children"])]
    dst = list(range(c["parents"], c["parents"] + len(src)))
    grow = dst if dst else list(range(c["parents"]))
    counts = _lengths(rng, len(grow), c["tokens_min"], c["tokens_max"])
    return lens, src, dst, grow, counts


def _compact_layout(c):
    rng = random.Random(c["mix"])
    base = _lengths(rng, c["base"], c["len_min"], c["len_max"])
    new = _lengths(rng, c["admitted"], c["len_min"], c["len_max"])
    gone = sorted(rng.sample(range(c["admitted"]), c["finished"]))
    return base, new, gone


def _pages(c):
    """(pages of the pool, columns of a table) for a step or a compaction."""
    page = c["page"]
    if c["kind"] == "step":
        lens, src, dst, grow, counts = _step_layout(c)
        have = sum(_up(n, page) for n in lens)
        more = sum(_up(n, page) + 1 for n in counts)
        return have + more + 8, _up(max(lens) + max(counts), page) + 1
    base, new, gone = _compact_layout(c)
    return sum(_up(n, page) for n in base + new) + 8, _up(max(base + new), page)


def _pool_bytes(c):
    return _pages(c)[0] * 2 * c["layers"] * c["kv_heads"] * c["page"] * c["d"] * 2


def work(c):
    token = c["kv_heads"] * c["d"] * 2                # bytes of one token's keys, or values, in one layer
    if c["kind"] == "attn":
        rows, lens, shared, ids, pages, cuts = _attn_layout(c)
        keys = sum(lens) - sum(s * c["page"] for s in shared)
        seen = sum(n * c["q_len"] - c["q_len"] * (c["q_len"] - 1) // 2 for n in lens)
        queries = c["batch"] * c["heads"] * c["q_len"]
        return {"bytes": 2 * token * keys + queries * (4 * c["d"] + 4), "flops": 4 * c["d"] * c["heads"] * seen}
    if c["kind"] == "step":
        lens, src, dst, grow, counts = _step_layout(c)
        copied = sum(lens[s] % c["page"] for s in src)
        return {"bytes": 4 * c["layers"] * token * (copied + sum(counts)), "flops": 0}
    base, new, gone = _compact_layout(c)
    page = c["page"]
    dead, at, live_at = set(gone), sum(_up(n, page) for n in base), []
    for i, n in enumerate(new):
        live_at += [] if i in dead else range(at, at + _up(n, page))
        at += _up(n, page)
    live = sum(_up(n, page) for n in base) + len(live_at)
    moved = sum(p >= live for p in live_at)
    return {"bytes": 4 * c["layers"] * token * page * moved + 4 * live, "flops": 0}


# ---------------------------------------------------------------- inputs

def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _ints(x, device):
    return torch.tensor(x, dtype=torch.int32, device=device)


def _normal(shape, gen, device):
    """Standard normal bf16, drawn in pieces (a pool is up to a few GB)."""
    out = torch.empty(shape, dtype=torch.bfloat16, device=device)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        flat[i:i + (1 << 28)].normal_(generator=gen)
    return out


def _table(rows, ids, seqs, columns, device):
    t = torch.full((seqs, columns), -1, dtype=torch.int32)
    for i, r in zip(ids, rows):
        t[i, :len(r)] = torch.tensor(r, dtype=torch.int32)
    return t.to(device)


def _cache(c, layers, pages, s):
    if own:
        from paper_2609_27373_amd.cache import PagedCache
        s["cache"] = PagedCache(layers, pages, c["page"], c["kv_heads"], c["d"], s["tables"].shape[0], s["tables"].shape[1], device=s["pool"].device,
                                pool=s["pool"], tables=s["tables"], lens=s["lens"], refs=s["refs"])
    return s


def prepare(c, seed):
    device = _device()
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    page = c["page"]
    if c["kind"] == "attn":
        rows, lens, shared, ids, pages, cuts = _attn_layout(c)
        seqs, columns = max(ids) + 1, max(len(r) for r in rows)
        s = dict(case=c, pool=_normal((2, pages, c["kv_heads"], page, c["d"]), gen, device), tables=_table(rows, ids, seqs, columns, device))
        all_lens = [0] * seqs
        for i, n in zip(ids, lens):
            all_lens[i] = n
        s["lens"], s["lens_host"], s["ids_host"] = _ints(all_lens, device), lens, ids
        refs = torch.zeros(pages, dtype=torch.int64)
        refs.index_add_(0, torch.tensor([p for r in rows for p in r]), torch.ones(sum(map(len, rows)), dtype=torch.int64))
        s["refs"] = refs.to(device, torch.int32)
        s["ids"] = _ints(ids, device) if c["slots"] else None
        s["shared"] = _ints(shared, device) if c["prefix"] else None
        s["q"] = _normal((c["batch"], c["heads"], c["q_len"], c["d"]), gen, device)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], dtype=torch.float32, device=device)
        return _cache(c, 1, pages, s)
    pages, columns = _pages(c)
    pool = _normal((2 * c["layers"], pages, c["kv_heads"], page, c["d"]), gen, device)
    if c["kind"] == "step":
        lens, src, dst, grow, counts = _step_layout(c)
        seqs = c["parents"] + len(dst)
    else:
        lens, new, gone = _compact_layout(c)
        seqs = c["base"] + c["admitted"]
    at, rows = 0, []
    for n in lens:
        rows.append(list(range(at, at + _up(n, page))))
        at += _up(n, page)
    tables = _table(rows, range(len(lens)), seqs, columns, device)
    refs = (torch.arange(pages, device=device) < at).to(torch.int32)
    s = dict(case=c, pool=pool, tables=tables, lens=_ints(lens + [0] * (seqs - len(lens)), device), refs=refs)
    if c["kind"] == "step":
        s["src"], s["dst"], s["grow"], s["counts"] = (_ints(x, device) for x in (src, dst, grow, counts))
        # what is dropped first: children of the last step, tokens past the accepted length
        s["back"] = _ints([0] * len(grow) if dst else lens, device)
        shape = (c["layers"], len(grow), c["kv_heads"], max(counts), c["d"])
        s["k"], s["v"] = _normal(shape, gen, device), _normal(shape, gen, device)
        s["done"], s["granted"] = torch.empty_like(s["dst"]), torch.empty_like(s["grow"])
        s["shared"] = torch.empty(seqs, dtype=torch.int32, device=device)
    else:
        s["new"] = _ints(list(range(c["base"], seqs)), device)
        s["gone"] = _ints([c["base"] + i for i in gone], device)
        s["counts"], s["granted"] = _ints(new, device), torch.empty_like(s["new"])
        s["live"] = torch.empty(1, dtype=torch.int32, device=device)
    return _cache(c, c["layers"], pages, s)


# ---------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    if c["kind"] == "attn":
        if own:
            s["cache"].attend(0, s["q"], s["out"], s["lse"], seq_ids=s["ids"], shared=s["shared"])
        else:
            _plain_attend(s)
        return {"o": s["out"], "lse": s["lse"]}
    if c["kind"] == "step":
        if own:
            a = s["cache"]
            a.trim(s["grow"], s["back"])
            if c["children"]:
                a.fork(s["src"], s["dst"], s["done"])
            a.reserve(s["grow"], s["counts"], s["granted"])
            for i in range(c["layers"]):
                a.append(i, s["k"][i], s["v"][i], s["grow"], s["granted"])
            a.shared(out=s["shared"])
        else:
            _plain_trim(s, s["grow"], s["back"])
            if c["children"]:
                _plain_fork(s)
            _plain_reserve(s, s["grow"])
            for i in range(c["layers"]):
                _plain_append(s, i)
            _plain_shared(s)
        out = {k: s[k] for k in ("pool", "tables", "lens", "refs", "granted", "shared")}
        return dict(out, done=s["done"]) if c["children"] else out
    if own:
        a = s["cache"]
        a.trim(s["new"])
        a.reserve(s["new"], s["counts"], s["granted"])
        a.trim(s["gone"])
        a.compact(s["live"])
    else:
        _plain_trim(s, s["new"], torch.zeros_like(s["new"]))
        _plain_reserve(s, s["new"])
        _plain_trim(s, s["gone"], torch.zeros_like(s["gone"]))
        _plain_compact(s)
    return {k: s[k] for k in ("pool", "tables", "lens", "refs", "granted", "live")}


# ---------------------------------------------------------------- the plain form

def _plain_attend(s):
    c = s["case"]
    page, q_len, kv, d = c["page"], c["q_len"], c["kv_heads"], c["d"]
    gq = c["heads"] // kv
    for b, (i, n) in enumerate(zip(s["ids_host"], s["lens_host"])):
        ids = s["tables"][i, :_up(n, page)].long()
        k, v = (s["pool"][x][ids].float().transpose(0, 1).reshape(kv, -1, d)[:, :n] for x in (0, 1))
        q = s["q"][b].float().view(kv, gq * q_len, d)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        if q_len > 1:                                 # token t sits at position n - q_len + t
            at = torch.arange(n - q_len, n, device=x.device).repeat(gq)
            x.masked_fill_(torch.arange(n, device=x.device)[None, :] > at[:, None], -math.inf)
        m = x.amax(-1, keepdim=True)
        p = torch.exp(x - m)
        z = p.sum(-1, keepdim=True)
        s["out"][b] = (torch.matmul(p, v) / z).view(c["heads"], q_len, d).to(torch.bfloat16)
        s["lse"][b] = (m + torch.log(z)).view(c["heads"], q_len)


def _used(s, lens):
    return (lens + s["case"]["page"] - 1) // s["case"]["page"]


def _plain_trim(s, ids, new_lens):
    ids = ids.long()
    old = s["lens"][ids]
    new = torch.minimum(old, new_lens)
    col = torch.arange(s["tables"].shape[1], device=ids.device)[None, :]
    rows = s["tables"][ids]
    drop = (col >= _used(s, new)[:, None]) & (col < _used(s, old)[:, None])
    s["refs"].index_add_(0, rows[drop].long(), torch.full_like(rows[drop], -1))
    s["tables"][ids] = torch.where(drop, -1, rows)
    s["lens"][ids] = new


def _plain_fork(s):
    src, dst = s["src"].long(), s["dst"].long()
    rows = s["tables"][src]
    s["tables"][dst] = rows
    s["lens"][dst] = s["lens"][src]
    named = rows[rows >= 0]
    s["refs"].index_add_(0, named.long(), torch.ones_like(named))
    s["done"].fill_(1)


def _plain_reserve(s, ids):
    """Room for s["counts"] tokens more: pages in ascending order from the free ones; a last page with others' names on it is copied."""
    page, ids = s["case"]["page"], ids.long()
    old, tables = s["lens"][ids], s["tables"]
    new = old + s["counts"]
    last = tables[ids, (torch.clamp(old, min=1) - 1).long() // page].long()
    copy = (old % page != 0) & (s["refs"][torch.clamp(last, min=0)] > 1)
    begin = _used(s, old) - copy.int()                # first column that gets a new page
    need = _used(s, new) - begin
    free = (s["refs"] == 0).nonzero().flatten()
    col = torch.arange(tables.shape[1], device=ids.device)[None, :]
    fill = (col >= begin[:, None]) & (col < _used(s, new)[:, None])
    slot = (torch.cumsum(need, 0) - need)[:, None] + col - begin[:, None]
    rows = tables[ids]
    got = free[slot[fill]]
    rows[fill] = got.int()
    tables[ids] = rows
    to = rows[torch.arange(len(ids), device=ids.device), (torch.clamp(old, min=1) - 1).long() // page].long()
    for i in range(page):                             # tokens of the copied pages
        w = copy & (i < old % page)
        s["pool"][:, to[w], :, i] = s["pool"][:, last[w], :, i]
    s["refs"].index_add_(0, last[copy], torch.full_like(last[copy], -1, dtype=torch.int32))
    s["refs"][got] = 1
    s["lens"][ids] = new
    s["granted"].copy_(s["counts"])


def _plain_append(s, layer):
    page, ids = s["case"]["page"], s["grow"].long()
    new, tokens = s["lens"][ids], s["k"].shape[3]
    t = torch.arange(tokens, device=ids.device)[None, :]
    put = t < s["granted"][:, None]
    at = (new - s["granted"])[:, None] + t
    seq = torch.arange(len(ids), device=ids.device)[:, None].expand(-1, tokens)[put]
    at, t = at[put].long(), t.expand(len(ids), -1)[put]
    pages = s["tables"][ids[seq], at // page].long()
    for x, what in ((0, "k"), (1, "v")):
        s["pool"][2 * layer + x][pages, :, at % page] = s[what][layer][seq, :, t]


def _plain_shared(s):
    """Leading pages that a sequence and the one before it both name and both fill."""
    page = s["case"]["page"]
    same = s["tables"][1:] == s["tables"][:-1]
    col = torch.arange(same.shape[1], device=same.device)[None, :]
    full = torch.minimum(s["lens"][1:], s["lens"][:-1]) // page
    run_ = torch.cumprod((same & (col < full[:, None])).int(), 1).sum(1)
    s["shared"].zero_()
    s["shared"][1:] = run_


def _plain_compact(s):
    used = s["refs"] > 0
    live = int(used.sum())
    src = used[live:].nonzero().flatten() + live
    dst = (~used[:live]).nonzero().flatten()
    s["pool"][:, dst] = s["pool"][:, src]
    to = torch.arange(used.numel(), dtype=torch.int32, device=used.device)
    to[src] = dst.int()
    named = s["tables"] >= 0
    s["tables"][named] = to[s["tables"][named].long()]
    s["refs"][dst] = s["refs"][src]
    s["refs"][src] = 0
    s["live"].fill_(live)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(c, seed):
    global own
    was, own = own, False
    s = prepare(c, seed)
    own = was
    page = c["page"]
    if c["kind"] == "attn":
        gq, q_len = c["heads"] // c["kv_heads"], c["q_len"]
        o = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
        lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=s["q"].device)
        tables = s["tables"].cpu().tolist()
        for b, (i, n) in enumerate(zip(s["ids_host"], s["lens_host"])):
            named = torch.tensor(tables[i][:_up(n, page)], device=o.device)
            for h in range(c["kv_heads"]):
                k, v = (s["pool"][x, named, h].reshape(-1, c["d"])[:n].double() for x in (0, 1))
                for t in range(q_len):
                    see = n - q_len + 1 + t
                    q = s["q"][b, h * gq:(h + 1) * gq, t].double()
                    x = (k[:see] @ q.t()) * c["d"] ** -0.5
                    z = torch.logsumexp(x, 0)
                    o[b, h * gq:(h + 1) * gq, t] = torch.exp(x - z).t() @ v[:see]
                    lse[b, h * gq:(h + 1) * gq, t] = z
        return {"o": o, "lse": lse}
    tables, lens, refs = s["tables"].cpu().tolist(), s["lens"].cpu().tolist(), s["refs"].cpu().tolist()
    pool = s["pool"]

    def trim(i, n):
        while _up(lens[i], page) > _up(n, page):
            j = _up(lens[i], page) - 1
            refs[tables[i][j]] -= 1
            tables[i][j] = -1
            lens[i] = j * page
        lens[i] = min(lens[i], n) if lens[i] < n else n

    def reserve(ids, counts):
        free = [p for p, n in enumerate(refs) if n == 0]
        named = list(refs)                            # counts before the call decide what is shared
        for i, n in zip(ids, counts):
            j = lens[i] // page
            if lens[i] % page and named[tables[i][j]] > 1:
                old, tables[i][j] = tables[i][j], free.pop(0)
                pool[:, tables[i][j], :, :lens[i] % page] = pool[:, old, :, :lens[i] % page]
                refs[old] -= 1
                refs[tables[i][j]] = 1
            for j in range(_up(lens[i], page), _up(lens[i] + n, page)):
                tables[i][j] = free.pop(0)
                refs[tables[i][j]] = 1
            lens[i] += n

    def done(**more):
        ints = dict(tables=tables, lens=lens, refs=refs, **more)
        return dict({k: torch.tensor(x, dtype=torch.int64) for k, x in ints.items()}, pool=pool)

    if c["kind"] == "step":
        base, src, dst, grow, counts = _step_layout(c)
        for a, b in zip(src, dst):
            tables[b], lens[b] = list(tables[a]), lens[a]
            for p in tables[b][:_up(lens[b], page)]:
                refs[p] += 1
        reserve(grow, counts)
        for e, (i, n) in enumerate(zip(grow, counts)):
            t = 0
            while t < n:                              # the stretch that lies in one page
                at = lens[i] - n + t
                m = min(n - t, page - at % page)
                for x, what in ((0, "k"), (1, "v")):
                    pool[x::2, tables[i][at // page], :, at % page:at % page + m] = s[what][:, e, :, t:t + m]
                t += m
        shared = [0]
        for i in range(1, len(lens)):
            j = 0
            while (j + 1) * page <= min(lens[i], lens[i - 1]) and tables[i][j] == tables[i - 1][j]:
                j += 1
            shared.append(j)
        out = done(granted=counts, shared=shared)
        return dict(out, done=torch.ones(len(dst), dtype=torch.int64)) if dst else out
    base, new, gone = _compact_layout(c)
    reserve(range(c["base"], c["base"] + len(new)), new)
    for i in gone:
        trim(c["base"] + i, 0)
    live = sum(n > 0 for n in refs)
    high = [p for p in range(live, len(refs)) if refs[p]]
    low = [p for p in range(live) if not refs[p]]
    to = dict(zip(high, low))
    for old, at in to.items():
        pool[:, at] = pool[:, old]
        refs[at], refs[old] = refs[old], 0
    tables = [[to.get(p, p) for p in row] for row in tables]
    return done(granted=new, live=[live])
