"""Positions of dma_cache_append_rope behind prefixes of any length, longer than a request of the shape can get among them: the formula of the
header, row_len - 1 behind the prefix, in extended precision."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from cache_harness import GpuCache, f64, normal
from oracle import cache_oracle as co, rope_oracle as ro
from paper_2508_02124_amd import binding as B
from test_gpu_cache_rope import CASES, ints
from test_gpu_rope import bound, frequencies

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_prefixes_longer_and_shorter_than_requests(gpu, case, interleaved, dtype):
    print(f"[case] positions {case} {interleaved} {dtype}", flush=True)
    n, H_q, H_kv, d, rot, ps = CASES[case]
    rng = np.random.default_rng(100 + case)
    n_reqs, pages = n + 2, n + 3
    cap = pages * ps
    cache, roomy, plain = (GpuCache(gpu, n_reqs, pages, m, ps, H_q, H_kv, d, dtype) for m in (pages, 1 << 12, pages))
    slots = rng.permutation(cap)[:n].astype(np.int32)
    slots[n // 2] = -1 if n > 1 else slots[n // 2]                     # a row without a place
    req = rng.permutation(n_reqs)[:n].astype(np.int32)
    length = rng.integers(1, 5000, n).astype(np.int32)
    prefix_len = np.array([cap - 1, cap, cap + 1, 100001, 2 ** 31 - 1, 0, -4, -2 ** 31], np.int32)
    of = rng.integers(-1, 9, n_reqs).astype(np.int32)                  # 8: out of range, as if none
    of[req[0]] = 3
    if n > 2:
        req[1], length[2], length[0] = n_reqs, -3, 0                   # no request; no length
    before = np.array([max(int(prefix_len[of[b]]), 0) if 0 <= b < n_reqs and 0 <= of[b] < 8 else 0 for b in req])
    positions = np.minimum(np.maximum(length.astype(np.int64) - 1, 0) + before, 2 ** 31 - 1)
    assert positions.max() > cap
    qkv = normal(gpu, case, n, H_q + 2 * H_kv, d, dtype=cache.type)
    q, K, V = qkv.split((H_q, H_kv, H_kv), 1)
    W, A, freqs = normal(gpu, 50 + case, H_q, d, scale=d ** -0.5), normal(gpu, 60 + case, H_q), frequencies(gpu, rot)
    Qo = torch.full((n, H_q, d), float("nan"), dtype=cache.type, device=gpu)
    s, pitch = ints(gpu, slots), qkv.stride(0)
    more = (ints(gpu, req), ints(gpu, length), 8, ints(gpu, prefix_len), ints(gpu, of), freqs, rot, interleaved)
    B.dma_cache_append_rope(cache.shape, n, q, pitch, K, pitch, V, pitch, W, A, None, s, *more, Qo, cache.pages)
    plain.append(K, V, s, W, A)
    k, v, z = cache.read(s)
    _, v0, z0 = plain.read(s)
    assert torch.equal(v, v0) and torch.equal(z, z0)
    ref, _ = ro.rotate(f64(K), positions, freqs.cpu().numpy(), interleaved)
    ref = co.quantise(ref)
    ref[slots < 0] = 0
    assert (f64(k) == ref).all()
    ref, size = ro.rotate(f64(q), positions, freqs.cpu().numpy(), interleaved)
    assert (np.abs(f64(Qo) - ref) <= bound(ref, size, dtype)).all()
    # pages that hold none of the rows are as they were; how many pages a request may have changes nothing
    free = torch.ones(pages, dtype=torch.bool, device=gpu)
    free[(s[s >= 0] // ps).long()] = False
    assert (cache.pages.view(pages, -1)[free] == 0xA5).all()
    Q2 = torch.empty_like(Qo)
    B.dma_cache_append_rope(roomy.shape, n, q, pitch, K, pitch, V, pitch, W, A, None, s, *more, Q2, roomy.pages)
    assert torch.equal(Q2, Qo) and torch.equal(roomy.pages, cache.pages)
    # scores given; queries in place, or none
    given, qc = normal(gpu, 70 + case, H_q, n), q.contiguous()
    B.dma_cache_append_rope(plain.shape, n, qc, H_q * d, K, pitch, V, pitch, None, None, given, s, *more, qc, plain.pages)
    k1, v1, z1 = plain.read(s)
    assert torch.equal(k1, k) and torch.equal(v1, v) and torch.equal(z1[:, s >= 0], given[:, s >= 0]) and torch.equal(qc, Qo)
    plain.pages.fill_(0xA5)
    B.dma_cache_append_rope(plain.shape, n, None, 0, K, pitch, V, pitch, W, A, None, s, *more, None, plain.pages)
    assert torch.equal(plain.pages, cache.pages)
