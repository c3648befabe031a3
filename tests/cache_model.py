"""The paged cache as the documentation defines it, in plain Python lists and
numpy: what the tests of the HIP path compare against.  Shares no code with
the library.  Pool entries are kept as the bf16 values' raw bits."""

import numpy as np


def up(x, y):
    return -(-x // y)


class Model:
    def __init__(self, planes, pages, page, kv_heads, d, seqs, max_pages, pool):
        self.planes, self.pages, self.page, self.kv, self.d = planes, pages, page, kv_heads, d
        self.seqs, self.max_pages = seqs, max_pages
        self.tables = [[-1] * max_pages for _ in range(seqs)]
        self.lens, self.refs = [0] * seqs, [0] * pages
        self.pool = np.array(pool, dtype=np.int16).reshape(planes, pages, kv_heads, page, d)

    def _firsts(self, ids):
        """Whether each entry is the first of its id, with an id that exists."""
        return [0 <= s < self.seqs and s not in ids[:i] for i, s in enumerate(ids)]

    def used(self, n):
        return up(n, self.page)

    def fork(self, src, dst):
        lens, tables = list(self.lens), [list(r) for r in self.tables]
        done = []
        for i, (a, b) in enumerate(zip(src, dst)):
            ok = 0 <= a < self.seqs and 0 <= b < self.seqs and b not in dst[:i] and a not in dst and lens[b] == 0
            done.append(int(ok))
            if ok:
                for j in range(self.used(lens[a])):
                    self.tables[b][j] = tables[a][j]
                    self.refs[tables[a][j]] += 1
                self.lens[b] = lens[a]
        return done

    def trim(self, ids, new_lens=None):
        for i, first in enumerate(self._firsts(ids)):
            s = ids[i]
            n = 0 if new_lens is None else max(new_lens[i], 0)
            if not first or n >= self.lens[s]:
                continue
            for j in range(self.used(n), self.used(self.lens[s])):
                self.refs[self.tables[s][j]] -= 1
                self.tables[s][j] = -1
            self.lens[s] = n

    def reserve(self, ids, counts):
        free = [p for p in range(self.pages) if self.refs[p] <= 0]
        refs = list(self.refs)
        at, granted = 0, []
        for i, first in enumerate(self._firsts(ids)):
            s, n = ids[i], counts[i]
            granted.append(0)
            if not first or n <= 0 or self.lens[s] + n > self.max_pages * self.page:
                continue
            old = self.lens[s]
            begin = self.used(old)
            copy = old % self.page != 0 and refs[self.tables[s][begin - 1]] > 1
            begin -= int(copy)
            need = self.used(old + n) - begin
            at += need
            if need and at > len(free):
                continue
            new = free[at - need:at]
            if copy:
                last, rows = self.tables[s][begin], old % self.page
                self.pool[:, new[0], :, :rows] = self.pool[:, last, :, :rows]
                self.refs[last] -= 1
            for j, p in enumerate(new):
                self.tables[s][begin + j] = p
                self.refs[p] = 1
            self.lens[s] = old + n
            granted[-1] = n
        return granted

    def append(self, layer, k, v, ids, counts):
        """k, v: int16 bits [n][kv][tokens][d]."""
        for e, s in enumerate(ids):
            n = min(max(counts[e], 0), k.shape[2])
            for t in range(n):
                pos = self.lens[s] - n + t if 0 <= s < self.seqs else -1
                if pos >= 0:
                    p = self.tables[s][pos // self.page]
                    self.pool[2 * layer, p, :, pos % self.page] = k[e, :, t]
                    self.pool[2 * layer + 1, p, :, pos % self.page] = v[e, :, t]

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        high = [p for p in range(live, self.pages) if self.refs[p] > 0]
        low = [p for p in range(live) if self.refs[p] <= 0]
        to = dict(zip(high, low))
        for a, b in to.items():
            self.pool[:, b] = self.pool[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.tables = [[to.get(p, p) for p in row] for row in self.tables]
        return live

    def shared(self, ids, min_pages=1):
        out = [0]
        for a, b in zip(ids, ids[1:]):
            n = 0
            if 0 <= a < self.seqs and 0 <= b < self.seqs:
                full = min(self.lens[a], self.lens[b]) // self.page
                while n < full and self.tables[a][n] == self.tables[b][n]:
                    n += 1
            out.append(n if n >= min_pages else 0)
        return out

    def counts_hold(self):
        """refs are the table entries' counts, columns past the last page -1."""
        refs = [0] * self.pages
        for row, n in zip(self.tables, self.lens):
            for j, p in enumerate(row):
                if j < self.used(n):
                    refs[p] += 1
                elif p != -1:
                    return False
        return refs == self.refs


def bf16_values(bits):
    """fp64 values of raw bf16 bits."""
    return (np.asarray(bits).astype(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def attend(q, k_pool, v_pool, tables, lens, ids, page, scale):
    """(o, lse, bound, lse_bound) in fp64 of the newest tokens q [batch][heads][q_len][d] over pools
    [pages][kv][page][d]: each row on its own over the positions it sees.

    bound: what a bf16 output may be off.  The output's rounding is half a
    step, 2^-8 |o|.  Probabilities enter the product with V rounded to bf16,
    2^-8 of each: 2^-8 A with A = sum p |v|.  The score is an fp32 sum of d
    exact products, off by at most E = scale d 2^-24 max_j sum |q k|, which
    changes a probability and the sum by a factor of at most e^E each; so do
    rescaled partial sums (an fp32 rounding a tile, counted with the exponentials'
    own error as 2^-16)."""
    batch, heads, q_len, d = q.shape
    pages, kv = k_pool.shape[:2]
    gq = heads // kv
    o, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    bound, lse_bound = np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(batch):
        s = ids[b]
        n = min(max(int(lens[s]), 0), tables.shape[1] * page) if 0 <= s < len(lens) else 0
        pos = np.arange(n)
        pg = tables[s][pos // page] if n else np.zeros(0, int)
        ok = (pg >= 0) & (pg < pages)
        for h in range(heads):
            for t in range(q_len):
                see = pos[ok & (pos <= n - q_len + t)]
                if see.size == 0:
                    continue
                k = k_pool[pg[see], h // gq, see % page]
                v = v_pool[pg[see], h // gq, see % page]
                x = scale * (k @ q[b, h, t])
                m = x.max()
                p = np.exp(x - m)
                z = p.sum()
                p /= z
                o[b, h, t] = p @ v
                lse[b, h, t] = m + np.log(z)
                e = scale * d * 2.0 ** -24 * (np.abs(k) @ np.abs(q[b, h, t])).max()
                a = p @ np.abs(v)
                bound[b, h, t] = 2.0 ** -8 * np.abs(o[b, h, t]) + (1 + 2.0 ** -8) * (2.0 ** -8 + 2 * e + 2.0 ** -16) * a
                lse_bound[b, h, t] = e + 2.0 ** -16 + 2.0 ** -22 * abs(lse[b, h, t])
    return o, lse, bound, lse_bound
