"""The paged cache's calls on a stream that is not the current one, and bounds on the rows' lengths through the objects."""
from __future__ import annotations

import pytest
import torch

from cache_harness import GpuCache, normal
from paper_2508_02124_amd import binding as B
from paper_2508_02124_amd.paged_cache import PagedCache
from paper_2508_02124_amd.torch_api import DynamicMaskAttention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,k", [((70, 33), 30), ((70, 33), 500), ((20000, 300), 1500)])
def test_every_call_runs_on_the_stream_that_it_is_given(gpu, lens, k):
    """assign, append, decode and read on a stream where their inputs appear only after a wait of some milliseconds: on any other stream
    they would work on the zeros that were there before."""
    H_q, H_kv, d, n = 4, 2, 64, sum(lens)
    K, V = normal(gpu, 1, n, H_kv, d).bfloat16(), normal(gpu, 2, n, H_kv, d).bfloat16()
    W, A, q = normal(gpu, 3, H_q, d, scale=0.125), -torch.ones(H_q, device=gpu), normal(gpu, 4, 2, H_q, d).bfloat16()
    change = torch.tensor(lens, dtype=torch.int32, device=gpu)

    def run(stream):
        cache = GpuCache(gpu, 2, 1300, 1260, 16, H_q, H_kv, d)
        given = [x.clone() for x in (K, V, q, change)]
        late = [torch.zeros_like(x) for x in given]
        rows = [torch.zeros(m, dtype=torch.int32, device=gpu) for m in (3, n, n, n, 2)]
        outs = [torch.zeros((2, H_q, d), dtype=torch.bfloat16, device=gpu), torch.zeros((H_q, 2), device=gpu), cache.ints(2, H_q, min(k, cache.cap)),
                torch.zeros_like(K), torch.zeros_like(V), torch.zeros((H_q, n), device=gpu)]
        size = B.dma_cache_decode_bytes(cache.shape, 2, k)
        ws = torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device=gpu)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            if stream:
                torch.cuda._sleep(10_000_000)
            for x, y in zip(late, given):
                x.copy_(y)
        B.dma_cache_assign(cache.shape, n, late[3], cache.lens, cache.table, cache.free, *rows, stream=stream)
        B.dma_cache_append(cache.shape, n, late[0], H_kv * d, late[1], H_kv * d, W, A, None, rows[3], cache.pages, stream=stream)
        B.dma_cache_decode(cache.shape, 2, k, 0.0, late[2], H_q * d, cache.pages, cache.table, None, cache.lens, *outs[:3], ws, size, stream=stream)
        B.dma_cache_read(cache.shape, n, rows[3], cache.pages, *outs[3:], stream=stream)
        torch.cuda.synchronize()
        full = [cache.lens, cache.table, *rows, *outs]
        B.dma_cache_reset(cache.shape, cache.lens.clone(), cache.table.clone(), cache.free, stream=stream)
        torch.cuda.synchronize()
        assert cache.free[0] == 1300
        return full

    want, got = run(None), run(torch.cuda.Stream())
    assert want[0].tolist() == list(lens) and (want[7] != 0).any()
    for x, y in zip(want, got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("max_len", [1, 100, 12288, 12289, 20000, 20001, 1 << 40])
def test_bounds_through_the_objects_change_nothing(gpu, max_len):
    """Bounds that hold and ones that do not, in PagedCache.decode and in a module's step."""
    H_q, H_kv, d, lens = 4, 2, 64, (20000, 12290, 40)
    cache = PagedCache(3, 600, H_q, H_kv, d, page_size=64, max_tokens=32768)
    module = DynamicMaskAttention(H_q, H_kv, d, 700, device=gpu)
    first, n = cache.assign(list(lens)), sum(lens)
    k, v = normal(gpu, 1, n, H_kv, d).bfloat16(), normal(gpu, 2, n, H_kv, d).bfloat16()
    cache.append(first.slots, k, v, W=module.W.detach(), A=module.A.detach())
    q = normal(gpu, 3, 3, H_q, d).bfloat16()
    for x, y in zip(cache.decode(q, 700), cache.decode(q, 700, max_len=max_len)):
        assert torch.equal(x, y)
    rows = cache.assign([1, 1, 1])
    new = [normal(gpu, i, 3, H_kv, d).bfloat16() for i in (4, 5)]
    want = module.step(q, *new, cache, rows)             # (the same rows go to the same places again)
    assert torch.equal(want, module.step(q, *new, cache, rows, max_len=max_len))


@pytest.mark.parametrize("cross_head", [False, True])
def test_steps_with_values_at_odd_places(gpu, cross_head):
    H_q, H_kv, d, n = 4, 2, 64, 37
    torch.manual_seed(3)
    module = DynamicMaskAttention(H_q, H_kv, d, 20, device=gpu, cross_head=cross_head)
    q, k, v = (normal(gpu, i, n, h, d).bfloat16() for i, h in ((1, H_q), (2, H_kv), (3, H_kv)))
    forms = [lambda x: x, lambda x: torch.cat((x.new_zeros(1), x.flatten()))[1:].view(x.shape), lambda x: torch.cat((x, x), 1)[:, x.shape[1]:],
             lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)]
    outs = []
    for form in forms:
        cache = PagedCache(1, 5, H_q, H_kv, d, page_size=16)
        rows = cache.assign([n])
        outs.append((module.step(form(q), form(k), form(v), cache, rows), *cache.read(rows.slots)))
    for out in outs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(outs[0], out))
