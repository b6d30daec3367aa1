"""A paged cache on the GPU beside the oracle's, for the tests."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache_oracle as co
from paper_2508_02124_amd import binding as B


class GpuCache:
    def __init__(self, dev, n_reqs, n_pages, max_pages, page_size, H_q, H_kv, d, dtype="bf16"):
        self.dev, self.type = dev, torch.bfloat16 if dtype == "bf16" else torch.float32
        self.H_q, self.H_kv, self.d, self.n_reqs = H_q, H_kv, d, n_reqs
        self.shape = B.make_cache_shape(n_reqs, n_pages, max_pages, page_size, H_q, H_kv, d,
                                        dtype=B.DMA_BF16 if dtype == "bf16" else B.DMA_F32)
        self.cap = max_pages * page_size
        self.pages = torch.full((B.dma_cache_bytes(self.shape),), 0xA5, dtype=torch.uint8, device=dev)
        self.lens, self.table, self.free = self.ints(n_reqs), self.ints(n_reqs, max_pages), self.ints(B.dma_cache_free_bytes(self.shape) // 4)
        B.dma_cache_reset(self.shape, self.lens, self.table, self.free)
        self.model = co.Pages(n_reqs, n_pages, max_pages, page_size)

    def ints(self, *shape):
        return torch.full(shape, -77, dtype=torch.int32, device=self.dev)

    def assign(self, change, n_rows):
        out = [self.ints(self.n_reqs + 1), self.ints(n_rows), self.ints(n_rows), self.ints(n_rows), self.ints(self.n_reqs)]
        c = torch.tensor(change, dtype=torch.int32, device=self.dev)
        B.dma_cache_assign(self.shape, n_rows, c, self.lens, self.table, self.free, *out)
        return out

    def append(self, K, V, slots, W=None, A=None, z=None, stream=None):
        B.dma_cache_append(self.shape, slots.numel(), K, K.stride(0), V, V.stride(0), W, A, z, slots, self.pages, stream)

    def read(self, slots):
        n = slots.numel()
        nan = float("nan")
        K = torch.full((n, self.H_kv, self.d), nan, dtype=self.type, device=self.dev)
        V, z = K.clone(), torch.full((self.H_q, n), nan, device=self.dev)
        B.dma_cache_read(self.shape, n, slots, self.pages, K, V, z)
        return K, V, z

    def decode(self, q, k, row_req, row_len, scale=0.0, table=None, stream=None):
        n = q.shape[0]
        o = torch.full((n, self.H_q, self.d), float("nan"), dtype=self.type, device=self.dev)
        lse = torch.full((self.H_q, n), float("nan"), device=self.dev)
        kept = self.ints(n, self.H_q, min(k, self.cap))
        size = B.dma_cache_decode_bytes(self.shape, n, k)
        ws = torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device=self.dev)
        B.dma_cache_decode(self.shape, n, k, scale, q, q.stride(0), self.pages, self.table if table is None else table, row_req,
                           row_len, o, lse, kept, ws, size, stream)
        return o, lse, kept


def normal(dev, seed, *shape, dtype=torch.float32, scale=1.0):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return (torch.randn(shape, generator=gen, device=dev) * scale).to(dtype)


def f64(t):
    return t.detach().double().cpu().numpy()
