"""Decode over the paged cache with more (row, head) pairs than the scratch has room for at once."""
from __future__ import annotations

import pytest
import torch

from cache_harness import GpuCache, normal
from paper_2508_02124_amd import binding as B
from test_gpu_cache import check_kept, check_rows, fill, request_slots

pytestmark = pytest.mark.gpu


# 4096 pairs have lists of 8192 keys each, more lists of 4096, and 8192 pairs fit the scratch: 64 rows and 65, 128 and 129, 300 (three
# launches).  "rising": keys of one slice only, "equal": ties, which no list holds.
@pytest.mark.parametrize("kind", ["ordinary", "rising", "equal"])
@pytest.mark.parametrize("n_rows", [64, 65, 128, 129, 300])
def test_many_pairs_share_the_scratch(gpu, kind, n_rows):
    print(f"[case] {n_rows} rows of 64 heads, {kind}", flush=True)
    lens, k, H, each = (29000, 12289, 12288, 300, 70000), 1500, 64, 20
    cache = GpuCache(gpu, 5, 2000, 1100, 64, H, 1, 64)
    fill(cache, lens, 8, "equal" if kind == "equal" else "ordinary")
    if kind == "rising":
        for b, n in enumerate(lens):
            slots = torch.from_numpy(request_slots(cache, b).astype("int32")).to(gpu)
            K, V, _ = cache.read(slots)
            cache.append(K, V, slots, z=torch.linspace(0.1, 0.9, n, device=gpu).expand(H, n).contiguous())
    rows = [(i % 5, lens[i % 5] - i // 5 % 7) for i in range(n_rows)]
    q = normal(gpu, 5, n_rows, H, 64).to(cache.type)
    req = torch.tensor([b for b, _ in rows], dtype=torch.int32, device=gpu)
    length = torch.tensor([n for _, n in rows], dtype=torch.int32, device=gpu)
    size = B.dma_cache_decode_bytes(cache.shape, n_rows, k)
    ws = torch.full((size + 65536,), 0xFF, dtype=torch.uint8, device=gpu)
    ws[size:] = 0x5A
    o, lse, kept = torch.zeros((n_rows, H, 64), dtype=cache.type, device=gpu), torch.zeros((H, n_rows), device=gpu), cache.ints(n_rows, H, k)
    for _ in range(2):                              # (the second time over what the first one left)
        kept.fill_(-77)
        B.dma_cache_decode(cache.shape, n_rows, k, 0.0, q, q.stride(0), cache.pages, cache.table, req, length, o, lse, kept, ws, size)
        assert (ws[size:] == 0x5A).all()
        for i in range(0, n_rows, each):            # calls of few rows, whose lists all have their room
            part = cache.decode(q[i:i + each], k, req[i:i + each], length[i:i + each])
            assert torch.equal(part[2], kept[i:i + each]), i
            assert torch.equal(part[0], o[i:i + each]) and torch.equal(part[1], lse[:, i:i + each]), i
    some = [0, n_rows // 2 - n_rows // 2 % 5 + 4, n_rows - 1]
    check_kept(cache, k, [rows[i] for i in some], kept[some])
    few = [i for i in some if rows[i][1] < 13000][:1] or [3]
    check_rows(cache, q[few], k, [rows[i] for i in few], (o[few], lse[:, few], kept[few]))


def test_captured_call_of_many_launches(gpu):
    """8320 pairs, two launches over the same scratch, in a graph: every replay equals the eager call, with eager calls over the same scratch
    between."""
    lens, k, H, n_rows = (29000, 300, 13000), 700, 64, 130
    cache = GpuCache(gpu, 3, 700, 460, 64, H, 1, 64)
    fill(cache, lens, 8)
    req = torch.arange(n_rows, device=gpu).remainder(3).int()
    length = (torch.tensor(lens, device=gpu)[req.long()] - torch.arange(n_rows, device=gpu) // 3).int()
    q = normal(gpu, 5, n_rows, H, 64).to(cache.type)
    size = B.dma_cache_decode_bytes(cache.shape, n_rows, k)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=gpu)

    def outputs():
        return torch.zeros((n_rows, H, 64), dtype=cache.type, device=gpu), torch.zeros((H, n_rows), device=gpu), cache.ints(n_rows, H, k)

    def call(out):
        B.dma_cache_decode(cache.shape, n_rows, k, 0.0, q, q.stride(0), cache.pages, cache.table, req, length, *out, ws, size)

    held, plain = outputs(), outputs()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call(held)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        call(plain)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, plain))
        for x in (*held, *plain):
            x.zero_()
        q.mul_(0.9)
        length.sub_(1)
