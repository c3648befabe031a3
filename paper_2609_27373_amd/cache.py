"""The keys and values that a generation keeps, in pages of one pool.

After a prompt's trajectory a model answers token by token: each step's keys
and values are kept, and the newest tokens attend to all of them.  PagedCache
owns the device buffers of the library's paged cache (tables, lengths,
reference counts, the pool of every layer's K and V) and calls the library on
the current stream.  A serving step is

    cache.fork(src, dst)                        # samples of a prompt share its pages
    granted = cache.reserve(ids, counts)        # room for the new tokens
    cache.append(layer, k, v, ids, granted)     # per layer
    cache.attend(layer, q, out, seq_ids=ids, shared=cache.shared(ids))
    cache.trim(ids, accepted)                   # drop drafts, or free finished ones

Ids, counts and lengths are int32 device tensors; nothing reads them back to
the host, so a step can be captured in a HIP graph: once the buffers exist (a
first call of attend() at each shape allocates its workspace) no call allocates
when its output tensors are given.  Graphs and streams that use one PagedCache
share its buffers and must run in order.
"""

from __future__ import annotations

import torch

from . import wise


class PagedCache:
    def __init__(self, layers, pages, page, kv_heads, head_dim, seqs, max_pages, device="cuda", pool=None, tables=None,
                 lens=None, refs=None):
        """`pool`, `tables`, `lens` and `refs` may be the caller's own buffers (of the layout in wise.h, in any
        valid state); those not given start out empty."""
        self.shape = wise.make_cache(pages, page, kv_heads, head_dim, 2 * layers, seqs, max_pages)
        n = wise.wise_cache_workspace_bytes(self.shape)
        if n == 0:
            raise ValueError(f"no such cache: layers {layers}, pages {pages}, page {page}, kv_heads {kv_heads}, "
                             f"head_dim {head_dim}, seqs {seqs}, max_pages {max_pages}")
        i32 = dict(dtype=torch.int32, device=device)
        self.pool = self._own(pool, (2 * layers, pages, kv_heads, page, head_dim), torch.bfloat16, "pool", lambda s: torch.zeros(
            s, dtype=torch.bfloat16, device=device))
        self.tables = self._own(tables, (seqs, max_pages), torch.int32, "tables", lambda s: torch.full(s, -1, **i32))
        self.lens = self._own(lens, (seqs,), torch.int32, "lens", lambda s: torch.zeros(s, **i32))
        self.refs = self._own(refs, (pages,), torch.int32, "refs", lambda s: torch.zeros(s, **i32))
        self.workspace = torch.empty(n, dtype=torch.uint8, device=device)
        self._planes = [self.pool[i] for i in range(2 * layers)]
        self._attend = {}

    @staticmethod
    def _own(t, shape, dtype, name, make):
        if t is None:
            return make(shape)
        if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} of shape {shape}")
        return t

    def _ints(self, n):
        return torch.empty(n, dtype=torch.int32, device=self.lens.device)

    def fork(self, src, dst, done=None):
        """Sequence dst[i] becomes a copy of src[i]; returns 1 per fork done, 0 per fork refused."""
        done = self._ints(src.numel()) if done is None else done
        wise.wise_cache_fork(self.shape, src, dst, self.tables, self.lens, self.refs, done)
        return done

    def trim(self, seq_ids, new_lens=None):
        """Drops the tokens from new_lens[i] on; without new_lens the sequences are freed."""
        wise.wise_cache_trim(self.shape, seq_ids, new_lens, self.tables, self.lens, self.refs)

    def reserve(self, seq_ids, counts, granted=None):
        """Room for counts[i] tokens more; returns the tokens granted (counts[i] or 0)."""
        granted = self._ints(seq_ids.numel()) if granted is None else granted
        wise.wise_cache_reserve(self.shape, seq_ids, counts, self.tables, self.lens, self.refs, granted, self.pool, self.workspace)
        return granted

    def append(self, layer, k, v, seq_ids, counts):
        """Writes the newest counts[i] tokens of each sequence in one layer; k, v: [n][kv_heads][tokens][head_dim]."""
        c = self.shape
        for t, name in ((k, "k"), (v, "v")):
            if t.dim() != 4 or tuple(t.shape[:2]) != (seq_ids.numel(), c.kv_heads) or t.shape[3] != c.head_dim:
                raise ValueError(f"{name} must be [{seq_ids.numel()}][{c.kv_heads}][tokens][{c.head_dim}], got {tuple(t.shape)}")
        if k.shape != v.shape:
            raise ValueError(f"k and v differ in shape: {tuple(k.shape)}, {tuple(v.shape)}")
        kp, vp = self.layer(layer)
        wise.wise_cache_append(c, k.shape[2], seq_ids, counts, k, v, self.tables, self.lens, kp, vp)

    def layer(self, layer):
        """The planes of one layer: (keys, values), [pages][kv_heads][page][head_dim]."""
        if not 0 <= layer < self.shape.planes // 2:
            raise ValueError(f"layer {layer} of {self.shape.planes // 2}")
        return self._planes[2 * layer], self._planes[2 * layer + 1]

    def compact(self, live=None):
        """Moves the pages in use to the front of the pool; returns their number (int32 [1], on the device)."""
        live = self._ints(1) if live is None else live
        wise.wise_cache_compact(self.shape, self.tables, self.refs, self.pool, live, self.workspace)
        return live

    def shared(self, seq_ids=None, min_pages=1, out=None):
        """Leading pages that each sequence has in common with the one before it (all sequences without seq_ids)."""
        batch = self.shape.seqs if seq_ids is None else seq_ids.numel()
        out = self._ints(batch) if out is None else out
        wise.wise_cache_shared(self.shape, batch, min_pages, seq_ids, self.tables, self.lens, out)
        return out

    def attend(self, layer, q, out, lse=None, seq_ids=None, shared=None, scale=0.0):
        """Attention of the newest tokens q [batch][heads][q_len][head_dim] of sequences seq_ids (0 .. batch-1
        without), after their keys and values were appended.  `shared` as shared() returns it."""
        c = self.shape
        if q.dim() != 4 or q.shape[3] != c.head_dim or out.shape != q.shape:
            raise ValueError(f"q and out must be [batch][heads][q_len][{c.head_dim}], got {tuple(q.shape)}, {tuple(out.shape)}")
        batch, heads, q_len = q.shape[:3]
        kp, vp = self.layer(layer)
        wise.wise_prefix_attn(c, wise.make_queries(batch, heads, q_len, scale), q, kp, vp, self.tables, self.lens, seq_ids, shared,
                              out, lse, self._attend_workspace(batch, heads, q_len))
        return out

    def _attend_workspace(self, batch, heads, q_len):
        # One per power of two of the batch, kept: a captured graph goes on using its own.
        key = (1 << max(batch - 1, 0).bit_length(), heads, q_len)
        if key not in self._attend:
            n = wise.wise_prefix_workspace_bytes(self.shape, wise.make_queries(*key))
            self._attend[key] = torch.empty(max(n, 1), dtype=torch.uint8, device=self.pool.device)
        return self._attend[key]
