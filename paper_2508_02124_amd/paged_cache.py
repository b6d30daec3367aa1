"""A paged 4-bit key/value cache as an object: its buffers, and the calls of a serving step on them.

Nothing here computes: buffers are allocated with torch and their addresses handed to the dma_cache_* entry points, whose
conventions hold (include/dma.h): fixed row capacities instead of lengths that the host would have to wait for, so that a
step runs without a synchronisation and can be captured in a graph.  There are no gradients: training goes through
torch_api.dynamic_mask_attention.  Calls run on the current stream of the cache's device; those of one cache must be ordered.

    cache = PagedCache(n_reqs=32, n_pages=4096, num_heads=32, num_kv_heads=8, head_dim=128)
    rows = cache.assign(change, n_rows)                 # places for the step's new tokens
    cache.append(rows.slots, k, v, W=W, A=A)            # their K, V and scores
    o, lse, kept = cache.decode(q, window, rows)        # attention from the new rows

With rotary positions, and requests behind prefixes that lie in the cache once (as requests of their own):

    shared = cache.prefixes([30, 31], of)               # requests 30 and 31 hold prefixes 0 and 1; of[b]: request b's, -1: none
    q = cache.append_rotary(rows, q, k, v, freqs, W=W, A=A, prefixes=shared)
    o, lse = cache.decode_prefix(q, window, rows, shared)
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B


class CacheRows(NamedTuple):
    """The rows of a step, all int32 on the cache's device (dma_cache_assign)."""
    cu_rows: torch.Tensor   # [n_reqs + 1]
    row_req: torch.Tensor   # [n_rows] request of a row, -1: none
    row_len: torch.Tensor   # [n_rows] keys that it sees, 0: none
    slots: torch.Tensor     # [n_rows] place of its token, -1: none
    status: torch.Tensor    # [n_reqs] 0: served, else binding.CACHE_NO_PAGES, CACHE_TOO_LONG, CACHE_NO_ROWS


class CachePrefixes(NamedTuple):
    """Prefixes that requests share, all int32 on the cache's device (dma_cache_decode_prefix)."""
    req: torch.Tensor   # [n_prefixes] the request that holds each
    len: torch.Tensor   # [n_prefixes] its tokens
    of: torch.Tensor    # [n_reqs] the prefix of each request, -1: none


class PagedCache:
    """n_reqs places for requests over a pool of n_pages pages; max_tokens: the longest that one request can get (default: the
    pool; a decode without max_len is the slower the longer it is).  dtype is that of k, v, q and o (bfloat16 or float32)."""

    def __init__(self, n_reqs, n_pages, num_heads, num_kv_heads, head_dim, page_size=64, max_tokens=None,
                 dtype=torch.bfloat16, device="cuda"):
        codes = {torch.bfloat16: B.DMA_BF16, torch.float32: B.DMA_F32}
        if dtype not in codes:
            raise TypeError(f"dtype must be bfloat16 or float32, got {dtype}")
        max_pages = n_pages if max_tokens is None else -(-int(max_tokens) // max(int(page_size), 1))
        self.shape = B.make_cache_shape(n_reqs, n_pages, max_pages, page_size, num_heads, num_kv_heads, head_dim,
                                        dtype=codes[dtype])
        B.dma_cache_describe(self.shape)                  # (raises for sizes that the library refuses)
        self.device, self.dtype = torch.device(device), dtype
        if self.device.type != "cuda":
            raise RuntimeError("the cache must live on the GPU: this library has no CPU path")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.pages = torch.empty(B.dma_cache_bytes(self.shape), dtype=torch.uint8, device=self.device)
        self.seq_lens = self._ints(n_reqs)
        self.block_table = self._ints(n_reqs, max_pages)
        self.free_list = self._ints(B.dma_cache_free_bytes(self.shape) // 4)
        self.reset()

    def reset(self):
        """Every request ends."""
        self._call(B.dma_cache_reset, self.seq_lens, self.block_table, self.free_list)

    def assign(self, change, n_rows=None):
        """Places for a step: request b grows by change[b] tokens or, below 0, gives its last -change[b] back.  change: int32
        tensor [n_reqs], or a sequence of ints; n_rows: capacity of the step's rows (a sequence's own number, if left out)."""
        if not isinstance(change, torch.Tensor):
            change = [int(c) for c in change]
            if n_rows is None:
                n_rows = sum(c for c in change if c > 0)
            change = torch.tensor(change, dtype=torch.int32, device=self.device)
        if n_rows is None:
            raise ValueError("n_rows is needed with a tensor (its sum is not looked at on the host)")
        self._check("change", change, (self.shape.n_reqs,), torch.int32)
        rows = CacheRows(self._ints(self.shape.n_reqs + 1), self._ints(n_rows), self._ints(n_rows), self._ints(n_rows),
                         self._ints(self.shape.n_reqs))
        self._call(B.dma_cache_assign, n_rows, change, self.seq_lens, self.block_table, self.free_list, *rows)
        return rows

    def append(self, slots, k, v, W=None, A=None, z=None):
        """k, v [n, num_kv_heads, head_dim] into their slots [n], with the scores of W [num_heads, head_dim] and A [num_heads], or
        with z [num_heads, n]."""
        self._check_append(slots, k, v, W, A, z)
        self._append(slots, k, v, None if W is None else self._aligned(W), A, z)

    def _check_append(self, slots, k, v, W, A, z):
        s, n = self.shape, slots.numel()
        self._check_values(slots, k, v)
        if (W is None) == (z is None) or (W is None) != (A is None):
            raise ValueError("the scores come from W and A, or are given as z")
        if z is None:
            self._check("W", W, (s.H_q, s.d), torch.float32)
            self._check("A", A, (s.H_q,), torch.float32)
        else:
            self._check("z", z, (s.H_q, n), torch.float32)

    def _append(self, slots, k, v, W, A, z):
        n, k, v = slots.numel(), self._rows(k), self._rows(v)
        self._call(B.dma_cache_append, n, k, k.stride(0), v, v.stride(0), W, A, z, slots, self.pages)

    def read(self, slots):
        """The tokens of slots [n]: k, v [n, num_kv_heads, head_dim] as the cache holds them and z [num_heads, n] (absent: 0 and -inf)."""
        s, n = self.shape, slots.numel()
        self._check("slots", slots, (n,), torch.int32)
        k = torch.empty((n, s.H_kv, s.d), dtype=self.dtype, device=self.device)
        v, z = torch.empty_like(k), torch.empty((s.H_q, n), dtype=torch.float32, device=self.device)
        self._call(B.dma_cache_read, n, slots, self.pages, k, v, z)
        return k, v, z

    def decode(self, q, keep_window, rows=None, softmax_scale=0.0, max_len=0):
        """Attention of q [n, num_heads, head_dim] over the cache: o, lse [num_heads, n] and the kept slots
        [n, num_heads, min(keep_window, longest request)].  rows: the step's (CacheRows), or (row_req, row_len); None: row r
        is request r with all its tokens.  max_len: the most keys that a row sees, where the host knows it (a matter of speed)."""
        return self._attend(q, *self._check_decode(q, keep_window, rows, softmax_scale, max_len), softmax_scale)

    def prefixes(self, req, of, length=None):
        """Prefixes held by the requests `req` (a sequence or int32 tensor), of[b] being that of request b (an index into them, -1: none;
        a sequence or int32 tensor [n_reqs]).  length: their tokens; left out: all that those requests have now.  Held by a request
        that is not there, a prefix has none, whatever its length.  (len of what this returns is a tensor of its own; a prefix that gets
        longer or shorter has it changed there.)"""
        ints = lambda x: x if isinstance(x, torch.Tensor) else torch.tensor([int(i) for i in x], dtype=torch.int32, device=self.device)
        req, of = ints(req), ints(of)
        given = length is not None
        length = ints(length) if given else req
        self._check_prefixes(CachePrefixes(req, length, of))
        there = (req >= 0) & (req < self.shape.n_reqs)
        if not given:
            length = self.seq_lens[req.long().clamp(0, self.shape.n_reqs - 1)]
        return CachePrefixes(req, length.where(there, 0).int(), of)

    def append_rotary(self, rows, q, k, v, freqs, W=None, A=None, z=None, prefixes=None, interleaved=False):
        """append of the step's rows with k, and q if there is one, turned to their positions (torch_api.rotary): a token's place in its
        request, behind the request's prefix.  freqs: float32 [rotated channels / 2].  Returns q [n, num_heads, head_dim] turned (None
        without one)."""
        self._check_rotary(rows, q, freqs, prefixes)
        self._check_append(rows.slots, k, v, W, A, z)
        return self._append_rotary(rows, q, k, v, freqs, None if W is None else self._aligned(W), A, z, prefixes, interleaved)

    def _append_rotary(self, rows, q, k, v, freqs, W, A, z, prefixes, interleaved):
        n, k, v = rows.slots.numel(), self._rows(k), self._rows(v)
        out = None if q is None else torch.empty((n, self.shape.H_q, self.shape.d), dtype=self.dtype, device=self.device)
        q = None if q is None else self._rows(q)
        shared = (0, None, None) if prefixes is None else (prefixes.req.numel(), prefixes.len, prefixes.of)
        self._call(B.dma_cache_append_rope, n, q, 0 if q is None else q.stride(0), k, k.stride(0), v, v.stride(0), W, A, z, rows.slots,
                   rows.row_req, rows.row_len, *shared, freqs, 2 * freqs.numel(), interleaved, out, self.pages)
        return out

    def decode_prefix(self, q, keep_window, rows, prefixes, softmax_scale=0.0, max_len=0, max_prefix=0):
        """decode where a row sees its request's prefix and then its own keys, and keeps the best of all of them: o and lse.  max_len,
        max_prefix: the most keys of its own that a row sees, and of a prefix, where the host knows them (a matter of speed)."""
        checked = self._check_decode(q, keep_window, rows, softmax_scale, max_len, prefixes, max_prefix)
        return self._attend_prefix(q, *checked, softmax_scale, prefixes, max_prefix)

    # ------------------------------------------------------------------
    def _ints(self, *shape):
        return torch.empty(shape, dtype=torch.int32, device=self.device)

    def _call(self, entry, *args):
        self._call_with(self.shape, entry, *args)

    def _call_with(self, shape, entry, *args):
        if torch.cuda.current_device() == self.device.index:
            entry(shape, *args)
        else:                                             # (the stream is that of the current device)
            with torch.cuda.device(self.device):
                entry(shape, *args)

    def _check(self, name, x, shape, dtype, whole=True):
        if x.device != self.device:
            raise RuntimeError(f"{name} must be on {self.device}, got {x.device}")
        if x.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {x.dtype}")
        if tuple(x.shape) != shape:
            raise ValueError(f"expected {name} {list(shape)}, got {list(x.shape)}")
        if whole and not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")

    def _check_values(self, slots, k, v):
        s, n = self.shape, slots.numel()
        self._check("slots", slots, (n,), torch.int32)
        for name, x in (("k", k), ("v", v)):
            self._check(name, x, (n, s.H_kv, s.d), self.dtype, whole=False)

    def _check_prefixes(self, prefixes):
        n = prefixes.req.numel()
        self._check("prefixes.req", prefixes.req, (n,), torch.int32)
        self._check("prefixes.len", prefixes.len, (n,), torch.int32)
        self._check("prefixes.of", prefixes.of, (self.shape.n_reqs,), torch.int32)

    def _check_rotary(self, rows, q, freqs, prefixes):
        s, n = self.shape, rows.slots.numel()
        if freqs.dim() != 1 or freqs.numel() % 8 or not 0 < 2 * freqs.numel() <= s.d:
            raise ValueError(f"expected freqs [m] with m a multiple of 8 and 2 m at most {s.d}, got {list(freqs.shape)}")
        self._check("freqs", freqs, tuple(freqs.shape), torch.float32)
        self._check("row_req", rows.row_req, (n,), torch.int32)
        self._check("row_len", rows.row_len, (n,), torch.int32)
        if q is not None:
            self._check("q", q, (n, s.H_q, s.d), self.dtype, whole=False)
        if prefixes is not None:
            self._check_prefixes(prefixes)

    def _check_decode(self, q, keep_window, rows, softmax_scale, max_len, prefixes=None, max_prefix=0):
        """The shape, window, row_req and row_len of a decode, or what it would raise, for a caller that has something to do before it.
        A window beyond all that a row can see (the longest request, with prefixes two of them), or a bound beyond the longest request, of
        whatever size, is one of just that."""
        s, n = self.shape, q.shape[0]
        longest = s.max_pages * s.page_size
        seen = longest if prefixes is None else min(2 * longest, 2 ** 31 - 1)
        window, bound = min(int(keep_window), seen), min(int(max_len), longest)
        name, n_prefixes = ("dma_cache_decode", 0) if prefixes is None else ("dma_cache_decode_prefix", prefixes.req.numel())
        if window <= 0 or bound < 0 or max_prefix < 0 or not softmax_scale >= 0.0:
            raise B.DmaError(B.DMA_EINVAL, name)
        if (n + n_prefixes + 8) * s.H_q * -(-min(window, longest) // 256) >= 1 << 22 or n_prefixes > 4096:
            raise B.DmaError(B.DMA_EUNSUPPORTED, name)
        if prefixes is not None:
            self._check_prefixes(prefixes)
        self._check("q", q, (n, s.H_q, s.d), self.dtype, whole=False)
        row_req, row_len = (None, self.seq_lens) if rows is None else (rows.row_req, rows.row_len) if isinstance(rows, CacheRows) else rows
        if rows is not None:
            self._check("row_req", row_req, (n,), torch.int32)
            self._check("row_len", row_len, (n,), torch.int32)
        if bound:
            s = B.make_cache_shape(s.n_reqs, s.n_pages, s.max_pages, s.page_size, s.H_q, s.H_kv, s.d, s.dtype, bound)
        return s, window, row_req, row_len

    def _attend(self, q, s, window, row_req, row_len, softmax_scale):
        q, n = self._rows(q), q.shape[0]
        o = torch.empty((n, s.H_q, s.d), dtype=self.dtype, device=self.device)
        lse = torch.empty((s.H_q, n), dtype=torch.float32, device=self.device)
        kept = self._ints(n, s.H_q, window)
        size = B.dma_cache_decode_bytes(s, n, window)
        ws = torch.empty(size, dtype=torch.uint8, device=self.device)
        self._call_with(s, B.dma_cache_decode, n, window, softmax_scale, q, q.stride(0), self.pages, self.block_table, row_req,
                        row_len, o, lse, kept, ws, size)
        return o, lse, kept

    def _attend_prefix(self, q, s, window, row_req, row_len, softmax_scale, prefixes, max_prefix):
        q, n, n_prefixes = self._rows(q), q.shape[0], prefixes.req.numel()
        max_prefix = min(int(max_prefix), s.max_pages * s.page_size)
        o = torch.empty((n, s.H_q, s.d), dtype=self.dtype, device=self.device)
        lse = torch.empty((s.H_q, n), dtype=torch.float32, device=self.device)
        size = B.dma_cache_decode_prefix_bytes(s, n, window, n_prefixes, max_prefix)
        ws = torch.empty(size, dtype=torch.uint8, device=self.device)
        self._call_with(s, B.dma_cache_decode_prefix, n, window, softmax_scale, q, q.stride(0), self.pages, self.block_table, row_req, row_len,
                        n_prefixes, max_prefix, prefixes.req, prefixes.len, prefixes.of, o, lse, ws, size)
        return o, lse

    @staticmethod
    def _aligned(x):
        return x if x.data_ptr() % 16 == 0 else x.clone()

    @staticmethod
    def _rows(x):
        """x, if its rows can be read where they are (whole, in steps of 8 elements, at addresses of 16 bytes); else a copy."""
        _, heads, d = x.shape
        fits = x.stride(2) == 1 and (heads == 1 or x.stride(1) == d) and x.stride(0) >= heads * d and x.stride(0) % 8 == 0
        return x if fits and x.data_ptr() % 16 == 0 else x.clone(memory_format=torch.contiguous_format)
