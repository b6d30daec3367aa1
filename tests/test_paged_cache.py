"""The cache object and the module's decoding step: refusals without a GPU, then whole runs against the entry points over plain
tensors."""
from __future__ import annotations

import os

import numpy as np
import pytest
import torch

from cache_harness import f64, normal
from paper_2508_02124_amd import binding as B
from paper_2508_02124_amd.paged_cache import PagedCache
from paper_2508_02124_amd.torch_api import DynamicMaskAttention


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g
        g.build()


def test_sizes_and_places_refused_without_a_gpu():
    for more in (dict(page_size=24), dict(head_dim=96), dict(num_heads=7), dict(n_reqs=0), dict(n_pages=0)):
        args = dict(n_reqs=2, n_pages=4, num_heads=4, num_kv_heads=2, head_dim=64)
        with pytest.raises(B.DmaError):
            PagedCache(**{**args, **more})
    with pytest.raises(TypeError):
        PagedCache(2, 4, 4, 2, 64, dtype=torch.float16)
    with pytest.raises(RuntimeError):
        PagedCache(2, 4, 4, 2, 64, device="cpu")


@pytest.mark.gpu
def test_arguments_refused(gpu):
    cache = PagedCache(2, 8, 4, 2, 64, page_size=16, max_tokens=50)
    rows = cache.assign([3, 2])
    k, W, A = normal(gpu, 1, 5, 2, 64).bfloat16(), normal(gpu, 2, 4, 64), normal(gpu, 3, 4)
    q = normal(gpu, 4, 5, 4, 64).bfloat16()
    for error, call in (
            (ValueError, lambda: cache.assign(torch.zeros(2, dtype=torch.int32, device=gpu))),
            (ValueError, lambda: cache.assign([1, 2, 3])),
            (TypeError, lambda: cache.assign(torch.zeros(2, dtype=torch.int64, device=gpu), 4)),
            (RuntimeError, lambda: cache.assign(torch.zeros(2, dtype=torch.int32), 4)),
            (TypeError, lambda: cache.append(rows.slots, k.float(), k, W=W, A=A)),
            (ValueError, lambda: cache.append(rows.slots, k[:4], k, W=W, A=A)),
            (ValueError, lambda: cache.append(rows.slots, k, k)),
            (ValueError, lambda: cache.append(rows.slots, k, k, W=W)),
            (ValueError, lambda: cache.append(rows.slots, k, k, W=W, A=A, z=torch.zeros((4, 5), device=gpu))),
            (ValueError, lambda: cache.append(rows.slots, k, k, z=torch.zeros((5, 4), device=gpu))),
            (ValueError, lambda: cache.append(rows.slots, k, k, z=torch.zeros((5, 4), device=gpu).t())),
            (TypeError, lambda: cache.read(rows.slots.long())),
            (ValueError, lambda: cache.decode(q[:, :3], 8, rows)),
            (ValueError, lambda: cache.decode(q[:4], 8, rows)),
            (B.DmaError, lambda: cache.decode(q, 8)),                       # five rows of two requests
            (B.DmaError, lambda: cache.decode(q, 0, rows)),
            (B.DmaError, lambda: cache.decode(q, 8, rows, softmax_scale=-1.0))):
        with pytest.raises(error):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_strides(gpu, dtype):
    """Rows that lie anyhow (transposed heads, odd offsets, every other channel) give what their contiguous copies give."""
    cache = PagedCache(2, 20, 4, 2, 64, page_size=16, dtype=dtype)
    rows = cache.assign([100, 37])
    n = 137
    k, v, q = (normal(gpu, i, n, h, 64).to(dtype) for i, h in ((1, 2), (2, 2), (3, 4)))
    W, A = normal(gpu, 4, 4, 64, scale=0.125), -torch.ones(4, device=gpu)
    cache.append(rows.slots, k, v, W=W, A=A)
    want, plain = cache.read(rows.slots), cache.decode(q, 30, rows)
    forms = [lambda x: x.transpose(0, 1).contiguous().transpose(0, 1),
             lambda x: torch.stack((x, x), -1).flatten(-2)[..., ::2],
             lambda x: torch.cat((x.flatten(1), x.flatten(1)[:, :1]), 1)[:, :-1].unflatten(1, x.shape[1:]),
             lambda x: torch.cat((x.new_zeros(1), x.flatten()))[1:].view(x.shape),
             lambda x: torch.cat((x, x, x), 1)[:, x.shape[1]:2 * x.shape[1]]]
    for form in forms:
        cache.pages.fill_(0xA5)
        cache.append(rows.slots, form(k), form(v), W=torch.cat((W.new_zeros(1), W.flatten()))[1:].view(W.shape), A=A)
        assert all(torch.equal(x, y) for x, y in zip(cache.read(rows.slots), want))
        assert all(torch.equal(x, y) for x, y in zip(cache.decode(form(q), 30, rows), plain))
    one = cache.assign([1, 0])
    cache.append(one.slots, form(k[:1]), form(v[:1]), W=W, A=A)
    assert torch.equal(cache.read(one.slots)[0], cache.read(rows.slots[:1])[0])


@pytest.mark.gpu
@pytest.mark.parametrize("cross_head", [False, True])
def test_module_steps_match_the_forward_over_the_cached_values(gpu, cross_head):
    """A module serves two requests (prompts, drafts, single tokens); at the end its outputs, row by row, are those of dma_mask_gen and
    dma_fwd over the rows read back, whose scores are the ones that the module's own forward selects on."""
    H_q, H_kv, d, window = 8, 2, 128, 60
    torch.manual_seed(3)
    module = DynamicMaskAttention(H_q, H_kv, d, window, device=gpu, cross_head=cross_head)
    cache = PagedCache(2, 60, H_q, H_kv, d, page_size=16, max_tokens=500)
    parts = {0: [], 1: []}
    for change in ([150, 40], [5, 1], [1, 1], [1, 260]):
        rows = cache.assign(change)
        n = sum(change)
        qkv = normal(gpu, n, n, H_q + 2 * H_kv, d).bfloat16()
        q, k, v = qkv.split((H_q, H_kv, H_kv), 1)
        o = module.step(q, k, v, cache, rows)
        assert not o.requires_grad and rows.status.tolist() == [0, 0]
        cu = rows.cu_rows.tolist()
        for b in (0, 1):
            parts[b].append((q[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]], rows.slots[cu[b]:cu[b + 1]], o[cu[b]:cu[b + 1]]))
    for b in (0, 1):
        q, v, slots, o = (torch.cat(x).contiguous() for x in zip(*parts[b]))
        n = q.shape[0]
        assert n == int(cache.seq_lens[b])
        kc, vc, z = cache.read(slots)
        shape = B.make_shape(n, 1, H_q, H_kv, d, window)
        cu = torch.tensor([0, n], dtype=torch.int32, device=gpu)
        expiry = torch.empty((H_q, n), dtype=torch.int32, device=gpu)
        mask = torch.empty(B.dma_mask_bytes(shape), dtype=torch.uint8, device=gpu)
        own = torch.empty_like(z)                       # the scores of the module's forward
        if cross_head:
            B.dma_scores_xhead(shape, v, module.W.detach(), module.A.detach(), own)
            assert torch.allclose(own, z, rtol=1e-5)
        else:
            B.dma_mask_gen(shape, v, module.W.detach(), module.A.detach(), cu, own, expiry, None, mask)
            assert torch.equal(own, z)
        B.dma_mask_gen(shape, None, None, None, cu, z, expiry, None, mask)
        O, LSE = torch.empty_like(q), torch.empty((H_q, n), device=gpu)
        B.dma_fwd(shape, q, kc, vc, z, expiry, mask, cu, O, LSE, None, 0)
        # the forward multiplies weights rounded to bf16 (half a step of 2^-8 each, a sum of their absolute values times that) and both
        # round their output once
        a, c = f64(O), f64(o)
        rms = np.sqrt((f64(vc) ** 2).mean())
        assert (np.abs(a - c) <= 2.0 ** -8 * (np.abs(a) + np.abs(c)) + 2.0 ** -8 * 3 * rms).all()


@pytest.mark.gpu
def test_captured_module_step(gpu):
    """A step in a graph: lengths, tables and the pool advance with every replay as they do eagerly."""
    H_q, H_kv, d = 4, 2, 64

    def run(captured):
        torch.manual_seed(5)
        module = DynamicMaskAttention(H_q, H_kv, d, 40, device=gpu)
        cache = PagedCache(3, 40, H_q, H_kv, d, page_size=16, max_tokens=160)
        first = cache.assign([70, 15, 1])
        k = normal(gpu, 1, 86, H_kv, d).bfloat16()
        cache.append(first.slots, k, k, W=module.W.detach(), A=module.A.detach())
        change = torch.ones(3, dtype=torch.int32, device=gpu)
        qkv = normal(gpu, 2, 3, H_q + 2 * H_kv, d).bfloat16()
        q, k, v = qkv.split((H_q, H_kv, H_kv), 1)
        step = lambda: module.step(q, k, v, cache, cache.assign(change, 3))
        torch.cuda.synchronize()
        if captured:
            graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            with torch.cuda.graph(graph, stream=side):
                held = step()
        out = []
        for i in range(20):                              # (requests cross page borders)
            if captured:
                graph.replay()
            else:
                held = step()
            torch.cuda.synchronize()
            out.append((held.clone(), cache.seq_lens.clone(), cache.block_table.clone()))
            qkv.mul_(0.9)
        return out

    for a, b in zip(run(False), run(True)):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.gpu
def test_two_caches_at_once(gpu):
    """Two caches on two streams, steps interleaved without waiting: each as if it were alone."""
    def make(seed, stream):
        with torch.cuda.stream(stream):
            cache = PagedCache(4, 300, 8, 2, 64, page_size=32)
            rows = cache.assign([700, 1500, 3, 40])
            n = 2243
            k, v = normal(gpu, seed, n, 2, 64).bfloat16(), normal(gpu, seed + 1, n, 2, 64).bfloat16()
            cache.append(rows.slots, k, v, W=normal(gpu, 3, 8, 64, scale=0.125), A=-torch.ones(8, device=gpu))
            return cache, normal(gpu, seed + 2, 4, 8, 64).bfloat16()

    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    both = [make(10, streams[0]), make(20, streams[1])]
    torch.cuda.synchronize()
    alone = []
    for (cache, q), s in zip(both, streams):
        with torch.cuda.stream(s):
            alone.append([x.clone() for x in cache.decode(q, 100)])
        torch.cuda.synchronize()
    got = [[], []]
    for _ in range(30):
        for i, ((cache, q), s) in enumerate(zip(both, streams)):
            with torch.cuda.stream(s):
                got[i].append(cache.decode(q, 100))
    torch.cuda.synchronize()
    for want, many in zip(alone, got):
        for one in many:
            assert all(torch.equal(x, y) for x, y in zip(want, one))
