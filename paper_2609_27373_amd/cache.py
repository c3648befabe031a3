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

Ids, counts and lengths are int32 tensors on the cache's device; nothing reads
them back to the host, so a step can be captured in a HIP graph.  attend() keeps one
workspace, which grows to the largest need seen; one that a graph has
captured is kept for it.  No other call allocates when its output tensors
are given.  Every call runs on the current stream of the cache's device, whichever
device is current.  Graphs and streams that use one PagedCache share its buffers and
must run in order.  A call on no sequences at all does nothing.

QuantCache is the same cache held in 8 or 4 bits: append() quantises, attend()
reads what was kept, read() gives it back in bf16, and everything else is as it was.
Where PagedCache takes 4 head_dim bytes a token and key-value head, it takes 2 (head_dim bits / 8 + head_dim / 32).
"""

from __future__ import annotations

import ctypes

import torch

from . import wise

_I32, _BF16, _F32 = torch.int32, torch.bfloat16, torch.float32

# The current stream's handle.  torch's public call builds a Stream object for it (1.2 us of the 7 of a call);
# its own generated code asks for the handle alone.
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
# The current device, which torch's public call first makes sure there is (as the cache's tensors have).
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class PagedCache:
    def __init__(self, layers, pages, page, kv_heads, head_dim, seqs, max_pages, device="cuda", pool=None, tables=None,
                 lens=None, refs=None):
        """`pool`, `tables`, `lens` and `refs` may be the caller's own buffers (of the layout in wise.h, in any
        valid state); those not given start out empty.  They stay the cache's for its life."""
        self.shape = wise.make_cache(pages, page, kv_heads, head_dim, 2 * layers, seqs, max_pages)
        self._c = ctypes.byref(self.shape)
        n = wise.wise_cache_workspace_bytes(self.shape)
        if n == 0:
            raise ValueError(f"no such cache: layers {layers}, pages {pages}, page {page}, kv_heads {kv_heads}, "
                             f"head_dim {head_dim}, seqs {seqs}, max_pages {max_pages}")
        i32 = dict(dtype=_I32, device=device)
        rows, dtype = self._page()
        self._pool = self._own(pool, (2 * layers, pages, kv_heads, *rows), dtype, "pool",
                               lambda s: torch.zeros(s, dtype=dtype, device=device))
        self._tables = self._own(tables, (seqs, max_pages), _I32, "tables", lambda s: torch.full(s, -1, **i32))
        self._lens = self._own(lens, (seqs,), _I32, "lens", lambda s: torch.zeros(s, **i32))
        self._refs = self._own(refs, (pages,), _I32, "refs", lambda s: torch.zeros(s, **i32))
        self.device = self._pool.device
        self._index, self._ordinal = self.device.index, self._pool.get_device()
        for t, name in ((self._tables, "tables"), (self._lens, "lens"), (self._refs, "refs")):
            if t.device != self.device:
                raise ValueError(f"{name} is on {t.device}, the pool on {self.device}")
        self._workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        self._attend = {}                       # bytes that attend() needs, by (batch, heads, q_len)
        self._room, self._held = None, {}       # its workspace (address, bytes, tensor); those that graphs use, by address
        # The buffers above, checked once and for all, as the C calls take them.
        self._state = tuple(t.data_ptr() for t in (self._tables, self._lens, self._refs))
        self._ws = (self._workspace.data_ptr(), n)
        plane = self._pool.numel() // self.shape.planes * self._pool.element_size()
        self._heads = (kv_heads, head_dim)
        self._planes = [(at, at + plane) for at in range(self._pool.data_ptr(), self._pool.data_ptr() + 2 * layers * plane, 2 * plane)]

    pool = property(lambda self: self._pool, doc="bf16 [2 * layers][pages][kv_heads][page][head_dim]")
    tables = property(lambda self: self._tables, doc="int32 [seqs][max_pages]")
    lens = property(lambda self: self._lens, doc="int32 [seqs]")
    refs = property(lambda self: self._refs, doc="int32 [pages]")

    # What differs where the pages hold something else: the entry points, their first arguments, a page of one head.
    _RESERVE, _APPEND, _COMPACT, _ATTEND = "wise_cache_reserve", "wise_cache_append", "wise_cache_compact", "wise_prefix_attn"
    _kind = ()

    def _page(self):
        return (self.shape.page, self.shape.head_dim), _BF16

    def _attend_bytes(self, queries):
        return wise.wise_prefix_workspace_bytes(self.shape, queries)

    @staticmethod
    def _own(t, shape, dtype, name, make):
        if t is None:
            return make(shape)
        if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} of shape {shape}")
        return t

    def _ints(self, n):
        return torch.empty(n, dtype=_I32, device=self.device)

    def _arg(self, t, dtype, name, numel):
        """The address of a call's tensor, or None."""
        if t is None:
            return None
        if t.dtype is dtype and t.get_device() == self._ordinal and t.is_contiguous() and t.numel() >= numel:
            return t.data_ptr()
        raise ValueError(f"{name} must be contiguous {dtype} on {self.device} of at least {numel} elements, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")

    def _call(self, fn, *args):
        index = self._index
        if index is None:
            raise ValueError("the cache is not on a GPU")
        entry = getattr(wise.load(), fn)
        stream = _stream(index)
        if _current() == index:
            status = entry(self._c, *args, stream)
        else:
            with torch.cuda.device(index):
                status = entry(self._c, *args, stream)
        if status != 0:
            raise wise.WiseError(status, fn)

    def fork(self, src, dst, done=None):
        """Sequence dst[i] becomes a copy of src[i]; returns 1 per fork done, 0 per fork refused."""
        n = src.numel()
        done = self._ints(n) if done is None else done
        self._call("wise_cache_fork", n, self._arg(src, _I32, "src", n), self._arg(dst, _I32, "dst", n), *self._state,
                   self._arg(done, _I32, "done", n))
        return done

    def trim(self, seq_ids, new_lens=None):
        """Drops the tokens from new_lens[i] on; without new_lens the sequences are freed."""
        n = seq_ids.numel()
        self._call("wise_cache_trim", n, self._arg(seq_ids, _I32, "seq_ids", n), self._arg(new_lens, _I32, "new_lens", n), *self._state)

    def reserve(self, seq_ids, counts, granted=None):
        """Room for counts[i] tokens more; returns the tokens granted (counts[i] or 0)."""
        n = seq_ids.numel()
        granted = self._ints(n) if granted is None else granted
        self._call(self._RESERVE, *self._kind, n, self._arg(seq_ids, _I32, "seq_ids", n), self._arg(counts, _I32, "counts", n), *self._state,
                   self._arg(granted, _I32, "granted", n), self._pool.data_ptr(), *self._ws)
        return granted

    def append(self, layer, k, v, seq_ids, counts):
        """Writes the newest counts[i] tokens of each sequence in one layer; k, v: [n][kv_heads][tokens][head_dim]."""
        n = seq_ids.numel()
        kp, vp, *args = self._rows(layer, k, v, seq_ids, counts, n)
        if n > 0:
            self._call(self._APPEND, *self._kind, n, k.shape[2], *args, *self._state[:2], kp, vp)

    def _rows(self, layer, k, v, seq_ids, counts, n):
        """Addresses of a layer's planes, and of the arguments that name rows of keys and values."""
        shape = tuple(k.shape)
        if len(shape) != 4 or shape[0] != n or (shape[1], shape[3]) != self._heads or v.shape != shape:
            c = self.shape
            raise ValueError(f"k and v must be [{n}][{c.kv_heads}][tokens][{c.head_dim}], got {shape}, {tuple(v.shape)}")
        return (*self._layer(layer), self._arg(seq_ids, _I32, "seq_ids", n), self._arg(counts, _I32, "counts", n),
                self._arg(k, _BF16, "k", 0), self._arg(v, _BF16, "v", 0))

    def _layer(self, layer):
        if not 0 <= layer < len(self._planes):
            raise ValueError(f"layer {layer} of {len(self._planes)}")
        return self._planes[layer]

    def layer(self, layer):
        """The planes of one layer: (keys, values), each as the pool without its first dimension."""
        self._layer(layer)
        return self._pool[2 * layer], self._pool[2 * layer + 1]

    def compact(self, live=None):
        """Moves the pages in use to the front of the pool; returns their number (int32 [1], on the device)."""
        live = self._ints(1) if live is None else live
        self._call(self._COMPACT, *self._kind, self._state[0], self._state[2], self._pool.data_ptr(), self._arg(live, _I32, "live", 1), *self._ws)
        return live

    def shared(self, seq_ids=None, min_pages=1, out=None):
        """Leading pages that each sequence has in common with the one before it (all sequences without seq_ids)."""
        batch = self.shape.seqs if seq_ids is None else seq_ids.numel()
        out = self._ints(batch) if out is None else out
        args = self._arg(seq_ids, _I32, "seq_ids", batch), *self._state[:2], self._arg(out, _I32, "out", batch)
        if batch > 0:
            self._call("wise_cache_shared", batch, min_pages, *args)
        return out

    def attend(self, layer, q, out, lse=None, seq_ids=None, shared=None, scale=0.0):
        """Attention of the newest tokens q [batch][heads][q_len][head_dim] of sequences seq_ids (0 .. batch-1
        without), after their keys and values were appended.  `shared` as shared() returns it."""
        if q.dim() != 4 or q.shape[3] != self.shape.head_dim or out.shape != q.shape:
            raise ValueError(f"q and out must be [batch][heads][q_len][{self.shape.head_dim}], got {tuple(q.shape)}, {tuple(out.shape)}")
        batch, heads, q_len = q.shape[:3]
        kp, vp = self._layer(layer)
        n, rows = q.numel(), batch * heads * q_len
        args = (self._arg(q, _BF16, "q", n), kp, vp, *self._state[:2], self._arg(seq_ids, _I32, "seq_ids", batch),
                self._arg(shared, _I32, "shared", batch), self._arg(out, _BF16, "out", n), self._arg(lse, _F32, "lse", rows))
        if batch > 0:
            self._call(self._ATTEND, *self._kind, ctypes.byref(wise.wise_queries(batch, heads, q_len, scale)), *args,
                       *self._attend_workspace(batch, heads, q_len))
        return out

    def _attend_workspace(self, batch, heads, q_len):
        key = (batch, heads, q_len)
        n = self._attend.get(key)
        if n is None:
            # For a power of two of sequences, so that a growing batch grows it seldom (or for the batch itself, where
            # that many more are past a limit).
            sizes = ((1 << max(batch - 1, 0).bit_length(), heads, q_len), key)
            n = next((x for x in (self._attend_bytes(wise.make_queries(*k)) for k in sizes) if x > 0), 0)
            if n == 0:
                return self._ws                 # for the call to refuse
            self._attend[key] = n
        capturing = self._index is not None and _stream(self._index) != 0 and self._capturing()   # the default stream can't be captured
        if self._room is None or self._room[1] < n:
            old, ws = self._room, torch.empty(n, dtype=torch.uint8, device=self.device)
            self._room = (ws.data_ptr(), n, ws)
            if old is not None and capturing:
                self._held[old[0]] = old[2]
            elif old is not None and ws.is_cuda:
                # Its memory may go to others once this call's stream is here: calls of a cache run in order, so
                # whatever used it, on any stream, has ended by then.
                old[2].record_stream(torch.cuda.current_stream(self.device))
        if capturing:
            self._held[self._room[0]] = self._room[2]
        return self._room[:2]

    def _capturing(self):
        with torch.cuda.device(self._index):
            return torch.cuda.is_current_stream_capturing()


class QuantCache(PagedCache):
    """A PagedCache whose keys and values are held in `bits` (8 or 4): 32 dims of a token's head share a power of two
    as their scale, a value is an E4M3 or E2M1 multiple of it (wise.h says which, and where the bytes lie)."""

    _RESERVE, _APPEND, _COMPACT, _ATTEND = "wise_qcache_reserve", "wise_qcache_append", "wise_qcache_compact", "wise_qcache_attn"

    def __init__(self, layers, pages, page, kv_heads, head_dim, seqs, max_pages, bits=4, device="cuda", pool=None, tables=None,
                 lens=None, refs=None):
        """As PagedCache; a pool is uint8 [2 * layers][pages][kv_heads][bytes of a page]."""
        if bits not in (4, 8):
            raise ValueError(f"bits must be 4 or 8, got {bits!r}")
        self.bits, self._kind = bits, (bits,)
        super().__init__(layers, pages, page, kv_heads, head_dim, seqs, max_pages, device, pool, tables, lens, refs)

    pool = property(lambda self: self._pool, doc="uint8 [2 * layers][pages][kv_heads][bytes of a page]")

    def _page(self):
        return (wise.wise_qcache_page_bytes(self.shape, self.bits),), torch.uint8

    def _attend_bytes(self, queries):
        return wise.wise_qcache_workspace_bytes(self.shape, self.bits, queries)

    def read(self, layer, k, v, seq_ids, counts, starts=None):
        """Positions starts[i] .. starts[i] + counts[i] - 1 (from 0 without starts) of each sequence in one layer, into
        k, v: bf16 [n][kv_heads][tokens][head_dim]; other rows stay as they are."""
        n = seq_ids.numel()
        kp, vp, ids, counts, k_to, v_to = self._rows(layer, k, v, seq_ids, counts, n)
        first = self._arg(starts, _I32, "starts", n)
        if n > 0:
            self._call("wise_qcache_read", self.bits, n, k.shape[2], ids, counts, first, kp, vp, *self._state[:2], k_to, v_to)
        return k, v
