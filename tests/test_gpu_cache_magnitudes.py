"""Rows of all magnitudes, subnormal and largest ones among them, through the cache: exactly the values of the definition."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from cache_harness import GpuCache, f64
from oracle import cache_oracle as co
from test_cache_error_bound import blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low,high", [(2.0 ** -149, 2.0 ** -120), (2.0 ** -130, 2.0 ** -122), (2.0 ** -20, 2.0 ** 20), (2.0 ** 120, 2.0 ** 128)])
def test_values_of_all_magnitudes(gpu, dtype, low, high):
    x, _ = blocks(low, high, 7, 4096)
    n = len(x) // 4                                  # rows of two heads of 64 channels, four blocks each
    cache = GpuCache(gpu, 1, n // 16 + 1, n // 16 + 1, 16, 2, 2, 64, dtype)
    K = torch.from_numpy(x[:4 * n].reshape(n, 2, 64)).to(gpu, torch.float32).to(cache.type)
    K = torch.where(torch.isfinite(K), K, torch.zeros_like(K))     # (bf16: the largest round to infinity)
    V = K.flip(0).contiguous()
    slots = torch.arange(n, dtype=torch.int32, device=gpu)
    cache.append(K, V, slots, z=torch.zeros((2, n), device=gpu))
    gK, gV, _ = cache.read(slots)
    for got, given in ((gK, K), (gV, V)):
        got, want = f64(got), co.quantise(f64(given))
        assert (got == want).all(), (np.argwhere(got != want)[:3], f64(given)[got != want][:3], got[got != want][:3], want[got != want][:3])
