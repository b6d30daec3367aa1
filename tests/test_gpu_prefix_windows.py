"""Windows longer than a request can get, behind prefixes, through PagedCache and DynamicMaskAttention, against the oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from cache_harness import f64, normal
from paper_2508_02124_amd.paged_cache import PagedCache
from paper_2508_02124_amd.torch_api import DynamicMaskAttention
from test_gpu_cache_prefix import Shared

pytestmark = pytest.mark.gpu


class Held(Shared):
    """What the rows of one request behind one prefix see, as the cache holds it."""

    def __init__(self, cache, H_q, H_kv, d, prefix, own):
        class Sizes:
            pass
        self.cache = Sizes()
        self.cache.H_q, self.cache.H_kv, self.cache.d, self.cache.type = H_q, H_kv, d, cache.dtype
        parts = [[f64(x) for x in cache.read(slots)] for slots in (prefix, own)]
        self.all = [np.concatenate(x, axis) for x, axis in zip(zip(*parts), (0, 0, 1))]
        self.before = prefix.numel()

    def keys(self, b, n):
        K, V, z = self.all
        return K[:self.before + n], V[:self.before + n], z[:, :self.before + n]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("window", [255, 256, 257, 300, 399, 490, 10 ** 9])
def test_windows_between_one_request_and_two(gpu, window, dtype):
    H_q, H_kv, d, P, m = 4, 2, 64, 250, 240
    torch.manual_seed(1)
    cache = PagedCache(3, 40, H_q, H_kv, d, page_size=16, max_tokens=256, dtype=dtype, device=gpu)
    layer = DynamicMaskAttention(H_q, H_kv, d, window, device=gpu)
    split = lambda seed, n: normal(gpu, seed, n, H_q + 2 * H_kv, d, dtype=dtype).split((H_q, H_kv, H_kv), 1)
    first = cache.assign([0, 0, P])
    layer.step(*split(1, P), cache, first)
    shared = cache.prefixes([2], [-1, 0, -1])
    rows = cache.assign([0, m, 0])
    q, k, v = split(2, m)
    o = layer.step(q, k, v, cache, rows, prefixes=shared)
    got = cache.decode_prefix(q, window, rows, shared)
    assert torch.equal(got[0], o)
    held = Held(cache, H_q, H_kv, d, first.slots, rows.slots)
    some = [0, 4, 5, 6, 7, 49, 50, 51, 148, 149, 150, 238, 239]
    at = torch.tensor(some, device=gpu)
    held.check(q[at], window, [(1, r + 1) for r in some], (got[0][at], got[1][:, at]))
