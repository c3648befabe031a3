"""The paged cache's calls together, as a generation uses them: prompts, samples
forked from them, drafted tokens checked and partly dropped, requests that end,
compaction, and at every step the attention of the newest tokens over what the
plain model says is kept; then a whole step captured in a HIP graph."""

import random

import numpy as np
import pytest
import torch

from cache_model import Model, attend, bf16_values
from paper_2609_27373_amd.cache import PagedCache
from parity_util import say

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server:
    """Both sides of a small generation: layers of the cache on the GPU, the model beside it."""

    def __init__(self, seed, layers=2, kv=2, gq=4, d=64, page=16, pages=120, seqs=14, max_pages=40):
        self.g = torch.Generator().manual_seed(seed)
        self.kv, self.gq, self.d, self.layers = kv, gq, d, layers
        self.cache = PagedCache(layers, pages, page, kv, d, seqs, max_pages)
        self.model = Model(2 * layers, pages, page, kv, d, seqs, max_pages, np.zeros((2 * layers, pages, kv, page, d), np.int16))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g).to(torch.bfloat16)

    def feed(self, ids, counts):
        """Room and keys and values for counts[i] new tokens; returns what was granted."""
        got = self.cache.reserve(ints(ids), ints(counts))
        want = self.model.reserve(ids, counts)
        assert got.cpu().tolist() == want
        for layer in range(self.layers):
            k, v = (self.normal(len(ids), self.kv, max(counts), self.d) for _ in range(2))
            self.cache.append(layer, k.cuda(), v.cuda(), ints(ids), got)
            self.model.append(layer, k.view(torch.int16).numpy(), v.view(torch.int16).numpy(), ids, want)
        return want

    def look(self, ids, q_len, layer):
        """Attention of the newest q_len tokens of a batch, with and without sharing, against the model's cache."""
        m, c = self.model, self.cache
        shared = c.shared(ints(ids))
        assert shared.cpu().tolist() == m.shared(ids)
        q = self.normal(len(ids), self.kv * self.gq, q_len, self.d)
        f64 = lambda x: bf16_values(x)  # noqa: E731
        scale = float(np.float32(1 / np.sqrt(self.d)))
        o, z, bound, zb = attend(f64(q.view(torch.int16).numpy()), f64(m.pool[2 * layer]), f64(m.pool[2 * layer + 1]),
                                 np.array(m.tables), np.array(m.lens), ids, m.page, scale)
        for sh in (shared, None):
            out, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:3], device="cuda")
            c.attend(layer, q.cuda(), out, lse, seq_ids=ints(ids), shared=sh)
            assert np.all(np.abs(out.double().cpu().numpy() - o) <= bound)
            some = ~np.isneginf(z)
            got = lse.double().cpu().numpy()
            assert np.array_equal(np.isneginf(got), ~some) and np.all(np.abs(got[some] - z[some]) <= zb[some])

    def same(self):
        m, c = self.model, self.cache
        assert c.lens.cpu().tolist() == m.lens and c.refs.cpu().tolist() == m.refs and c.tables.cpu().tolist() == m.tables
        assert np.array_equal(c.pool.view(torch.int16).cpu().numpy(), m.pool) and m.counts_hold()


@pytest.mark.parametrize("seed,shape", [(0, {}), (1, dict(page=32, d=96, gq=1, kv=3)), (2, dict(page=128, d=128, pages=40, max_pages=8)),
                                        (3, dict(page=64, d=64, gq=8, kv=1, pages=60))])
def test_generation(gpu_lib, seed, shape):
    rng = random.Random(seed)
    s = Server(seed, **shape)
    m, c = s.model, s.cache
    say(f"generation {seed}: {shape}")
    busy = []
    for step in range(12):
        idle = [i for i in range(m.seqs) if i not in busy]
        if len(busy) < 4 and len(idle) > 4:           # a prompt and its samples
            root, n = idle[0], rng.randint(1, 4)
            if s.feed([root], [rng.randint(1, 150)])[0]:
                assert c.fork(ints([root] * n), ints(idle[1:1 + n])).cpu().tolist() == m.fork([root] * n, idle[1:1 + n])
                busy += [root] + idle[1:1 + n]
        q_len = rng.choice((1, 1, 3))
        got = s.feed(busy, [q_len] * len(busy))       # drafts; refused where the pool is full
        s.look(busy, q_len, step % s.layers)
        keep = [m.lens[i] - rng.randint(0, q_len - 1) if n else m.lens[i] for i, n in zip(busy, got)]
        c.trim(ints(busy), ints(keep))
        m.trim(busy, keep)
        if len(busy) > 8 or step % 4 == 3:            # some end, the pool is compacted
            gone = rng.sample(busy, len(busy) // 2)
            c.trim(ints(gone))
            m.trim(gone)
            busy = [i for i in busy if i not in gone]
            assert int(c.compact().item()) == m.compact()
        s.same()
        if busy:
            s.look(busy, 1, 0)


def test_a_step_in_a_graph(gpu_lib):
    """Trim, fork, reserve, append, shared and attend of a step captured once, replayed between eager steps."""
    s = Server(7)
    m, c = s.model, s.cache
    s.feed([0, 1], [70, 33])
    src, dst, counts = [0, 0, 1], [5, 6, 7], [3, 3, 3]
    dsrc, ddst, dcounts = ints(src), ints(dst), ints(counts)
    done, granted, shared = (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(3))
    k, v = (s.normal(3, s.kv, 3, s.d) for _ in range(2))
    kd, vd, q = k.cuda(), v.cuda(), s.normal(3, s.kv * s.gq, 3, s.d)
    qd = q.cuda()
    out, lse = torch.empty_like(qd), torch.empty(qd.shape[:3], device="cuda")

    def step():
        c.trim(ddst)
        c.fork(dsrc, ddst, done)
        c.reserve(ddst, dcounts, granted)
        for layer in range(s.layers):
            c.append(layer, kd, vd, ddst, granted)
        c.shared(ddst, out=shared)
        c.attend(1, qd, out, lse, seq_ids=ddst, shared=shared)

    c.attend(1, qd, out, lse, seq_ids=ddst, shared=None)      # its workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    f64 = lambda x: bf16_values(x.view(torch.int16).numpy())  # noqa: E731
    for rep in range(4):
        out.fill_(float("nan"))
        graph.replay()
        m.trim(dst)
        m.fork(src, dst)
        want = m.reserve(dst, counts)
        for layer in range(s.layers):
            m.append(layer, k.view(torch.int16).numpy(), v.view(torch.int16).numpy(), dst, want)
        torch.cuda.synchronize()
        s.same()
        assert shared.cpu().tolist() == m.shared(dst) and granted.cpu().tolist() == want
        o, z, bound, zb = attend(f64(q), bf16_values(m.pool[2]), bf16_values(m.pool[3]), np.array(m.tables), np.array(m.lens), dst, m.page,
                                 float(np.float32(1 / np.sqrt(s.d))))
        assert np.all(np.abs(out.double().cpu().numpy() - o) <= bound) and np.all(np.abs(lse.double().cpu().numpy() - z) <= zb)
        eager = torch.empty_like(out)
        c.attend(1, qd, eager, seq_ids=ddst, shared=shared)
        assert torch.equal(eager, out)
        s.feed([0], [1])                              # the prompt grows between replays
