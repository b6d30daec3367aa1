"""dma_cache_append_rope on the GPU: the codes of the turned rows, bit for bit, and the turned queries."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co, rope_oracle as ro
from paper_2508_02124_amd import binding as B
from cache_harness import GpuCache, f64, normal
from test_gpu_rope import bound, frequencies

pytestmark = pytest.mark.gpu


def ints(dev, values):
    return torch.tensor(values, dtype=torch.int32, device=dev)


CASES = [  # rows, H_q, H_kv, d, rot, page size
    (1, 32, 8, 128, 128, 64), (3, 4, 2, 64, 64, 16), (13, 6, 2, 128, 48, 32), (9, 5, 1, 256, 256, 128), (37, 3, 3, 256, 64, 256),
    (130, 16, 16, 64, 16, 16), (17, 24, 2, 128, 112, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_codes_scores_and_queries(gpu, case, interleaved, dtype):
    n, H_q, H_kv, d, rot, ps = CASES[case]
    rng = np.random.default_rng(case)
    n_reqs, pages = n + 2, n + 3
    cache, plain = (GpuCache(gpu, n_reqs, pages, pages, ps, H_q, H_kv, d, dtype) for _ in range(2))
    slots = rng.permutation(pages * ps)[:n].astype(np.int32)
    slots[n // 2] = -1 if n > 1 else slots[n // 2]                     # a row without a place
    req = rng.permutation(n_reqs)[:n].astype(np.int32)
    length = rng.integers(1, 5000, n).astype(np.int32)
    prefix_len = np.array([100001, pages * ps, 0, -4], np.int32)
    of = rng.integers(-1, 5, n_reqs).astype(np.int32)                 # 4: out of range, as if none
    if n > 2:
        req[0], length[0], length[1], of[req[2]] = -1, 0, -3, 0       # no request; no length
    cap = pages * ps
    before = np.array([np.clip(prefix_len[of[b]], 0, cap) if b >= 0 and 0 <= of[b] < 4 else 0 for b in req])
    positions = np.maximum(length - 1, 0) + before
    qkv = normal(gpu, case, n, H_q + 2 * H_kv, d, dtype=cache.type)
    q, K, V = qkv.split((H_q, H_kv, H_kv), 1)
    W, A, freqs = normal(gpu, 50 + case, H_q, d, scale=d ** -0.5), normal(gpu, 60 + case, H_q), frequencies(gpu, rot)
    Qo = torch.full((n, H_q, d), float("nan"), dtype=cache.type, device=gpu)
    s, pitch = ints(gpu, slots), qkv.stride(0)
    more = (ints(gpu, req), ints(gpu, length), 4, ints(gpu, prefix_len), ints(gpu, of), freqs, rot, interleaved)
    B.dma_cache_append_rope(cache.shape, n, q, pitch, K, pitch, V, pitch, W, A, None, s, *more, Qo, cache.pages)
    plain.append(K, V, s, W, A)
    k, v, z = cache.read(s)
    _, v0, z0 = plain.read(s)
    assert torch.equal(v, v0) and torch.equal(z, z0)
    # codes of the value in 64 bits: the two differ by 2^-52 of it, so only one in 10^12 could lie next to a border
    ref, _ = ro.rotate(f64(K), positions, freqs.cpu().numpy(), interleaved)
    ref = co.quantise(ref)
    ref[slots < 0] = 0
    assert (f64(k) == ref).all()
    ref, size = ro.rotate(f64(q), positions, freqs.cpu().numpy(), interleaved)
    assert (np.abs(f64(Qo) - ref) <= bound(ref, size, dtype)).all()
    # pages that hold none of the rows are as they were; scores given; queries in place, or none
    at = cache.pages.view(pages, -1)
    free = torch.ones(pages, dtype=torch.bool, device=gpu)
    free[(s[s >= 0] // ps).long()] = False
    assert (at[free] == 0xA5).all()
    given, qc = normal(gpu, 70 + case, H_q, n), q.contiguous()
    B.dma_cache_append_rope(plain.shape, n, qc, H_q * d, K, pitch, V, pitch, None, None, given, s, *more, qc, plain.pages)
    k1, v1, z1 = plain.read(s)
    assert torch.equal(k1, k) and torch.equal(v1, v) and torch.equal(z1[:, s >= 0], given[:, s >= 0]) and torch.equal(qc, Qo)
    plain.pages.fill_(0xA5)
    B.dma_cache_append_rope(plain.shape, n, None, 0, K, pitch, V, pitch, W, A, None, s, *more, None, plain.pages)
    assert torch.equal(plain.pages, cache.pages)


def test_position_0_is_the_plain_append(gpu):
    """Also where the values are of every size, infinite or no numbers; and without prefixes no request is read."""
    n, H_q, H_kv, d, ps = 64, 4, 2, 64, 16
    cache, plain = (GpuCache(gpu, 3, 8, 8, ps, H_q, H_kv, d, "f32") for _ in range(2))
    K = normal(gpu, 1, n, H_kv, d) * torch.exp2(torch.randint(-130, 127, (n, 1, 1), device=gpu).float())
    K[3, 0, 5], K[4, 1, 40], K[5, 0, 63], K[6] = float("nan"), float("inf"), -float("inf"), 0.0
    V, z, s = normal(gpu, 2, n, H_kv, d), normal(gpu, 3, H_q, n), torch.randperm(128, device=gpu)[:n].int()
    turned = K.clone()
    turned[4, 1, 16] = float("nan")      # the other half of channel 40's pair: x1 cos 0 - inf sin 0 = inf * 0 (channel 63 stays as it is)
    plain.append(turned, V, s, z=z)
    one = ints(gpu, [1] * n)
    B.dma_cache_append_rope(cache.shape, n, None, 0, K, H_kv * d, V, H_kv * d, None, None, z, s, None, one, 0, None, None, frequencies(gpu, 48), 48,
                            False, None, cache.pages)
    for x, y in zip(cache.read(s), plain.read(s)):
        assert torch.equal(x.view(torch.int32), y.view(torch.int32))


def test_values_on_the_borders_between_codes(gpu):
    """A turn by a half or quarter circle of values that are borders themselves; sums that only 64 bits tell from a border."""
    d, ps = 64, 16
    cache = GpuCache(gpu, 1, 4, 4, ps, 1, 1, d, "f32")
    rows, rng = 32, np.random.default_rng(2)
    K = np.zeros((rows, 1, d), np.float32)
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    K[:, 0, 0:32] = rng.choice(grid, (rows, 32)) * rng.choice([-1, 1], (rows, 32))
    K[:, 0, 32:] = rng.choice([0.0, 2.0 ** -20, -2.0 ** -30], (rows, 32))
    freqs = torch.full((32,), 2.0 ** -12, device=gpu)                 # (small angles: a border plus or minus little)
    length = np.arange(1, rows + 1, dtype=np.int32)
    Kt = torch.from_numpy(K).to(gpu)
    s = torch.arange(rows, device=gpu).int()
    B.dma_cache_append_rope(cache.shape, rows, None, 0, Kt, d, Kt, d, None, None, normal(gpu, 1, 1, rows), s, None, ints(gpu, length), 0, None, None,
                            freqs, d, False, None, cache.pages)
    ref, _ = ro.rotate(K, length - 1, freqs.cpu().numpy())
    assert (f64(cache.read(s)[0]) == co.quantise(ref)).all()


def test_graph_replays(gpu):
    n, H_q, H_kv, d, ps = 20, 4, 2, 128, 16
    cache, eager = (GpuCache(gpu, n, 64, 8, ps, H_q, H_kv, d) for _ in range(2))
    qkv = normal(gpu, 1, n, H_q + 2 * H_kv, d, dtype=torch.bfloat16)
    q, K, V = qkv.split((H_q, H_kv, H_kv), 1)
    W, A, freqs = normal(gpu, 2, H_q, d, scale=0.1), normal(gpu, 3, H_q), frequencies(gpu, d)
    length, prefix_len, of = ints(gpu, list(range(1, n + 1))), ints(gpu, [77]), ints(gpu, [0, -1] * (n // 2))
    slots = torch.arange(n, device=gpu).int() * ps
    outs = [torch.zeros((n, H_q, d), dtype=torch.bfloat16, device=gpu) for _ in range(2)]
    call = lambda c, out: B.dma_cache_append_rope(c.shape, n, q, qkv.stride(0), K, qkv.stride(0), V, qkv.stride(0), W, A, None, slots, None, length, 1,
                                                  prefix_len, of, freqs, d, False, out, c.pages)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(cache, outs[0])
    for seed in range(3):
        qkv.copy_(normal(gpu, 20 + seed, *qkv.shape, dtype=torch.bfloat16))
        length += 7
        prefix_len += 1
        call(eager, outs[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        assert all(torch.equal(a, b) for a, b in zip(cache.read(slots), eager.read(slots)))


def test_more_rows_than_a_launch_takes(gpu):
    n, d, ps = (1 << 22) + 21, 64, 256
    cache = GpuCache(gpu, 1, n // ps + 2, n // ps + 2, ps, 1, 1, d)
    K = normal(gpu, 1, 512, 1, d, dtype=torch.bfloat16).repeat(n // 512 + 1, 1, 1)[:n]
    freqs, slots = frequencies(gpu, d, 500000.0), torch.arange(n, device=gpu).int()
    length, z = slots + 1, torch.rand((1, n), device=gpu)
    q = torch.full((n + 3, 1, d), 5.0, dtype=torch.bfloat16, device=gpu)
    B.dma_cache_append_rope(cache.shape, n, K, d, K, d, K, d, None, None, z, slots, None, length, 0, None, None, freqs, d, True, q, cache.pages)
    at = torch.cat((torch.arange(0, 1 << 22, 99991), torch.arange((1 << 22) - 9, n))).to(gpu)
    k, v, zz = cache.read(slots[at])
    ref, size = ro.rotate(f64(K[at]), at.cpu().numpy(), freqs.cpu().numpy(), True)
    assert (f64(k) == co.quantise(ref)).all() and (f64(v) == co.quantise(f64(K[at]))).all() and torch.equal(zz, z[:, at])
    assert (np.abs(f64(q[at]) - ref) <= bound(ref, size, "bf16")).all() and (q[n:] == 5).all()


def test_lengths_at_the_ends_of_their_type(gpu):
    """Below 1: position 0, behind a prefix the prefix's length; the largest: at most 2^31 - 1, also behind a prefix."""
    n, d, low, high = 6, 64, -2 ** 31, 2 ** 31 - 1
    cache = GpuCache(gpu, n, 4, 4, 16, 2, 1, d, "f32")
    freqs, slots = frequencies(gpu, d), torch.arange(n, device=gpu).int()
    q, K = normal(gpu, 1, n, 2, d), normal(gpu, 2, n, 1, d)
    W, A = normal(gpu, 3, 2, d), normal(gpu, 4, 2)
    length, of = ints(gpu, [low, low, high, high, 0, -5]), ints(gpu, [-1, 0, -1, 0, 1, 1])
    out = torch.empty_like(q)
    B.dma_cache_append_rope(cache.shape, n, q, 2 * d, K, d, K, d, W, A, None, slots, None, length, 2, ints(gpu, [37, low]), of, freqs, d, False, out,
                            cache.pages)
    at = [0, 37, high - 1, min(high - 1 + 37, high), 0, 0]
    ref, size = ro.rotate(f64(q), at, freqs.cpu().numpy(), False)
    assert (np.abs(f64(out) - ref) <= bound(ref, size, "f32")).all()
    assert (f64(cache.read(slots)[0]) == co.quantise(ro.rotate(f64(K), at, freqs.cpu().numpy(), False)[0])).all()
