"""DynamicMaskAttention.step: what is refused is refused before any kernel reads an address (on the CPU, with the launches recorded)."""
from __future__ import annotations

import pytest
import torch

from paper_2508_02124_amd import binding as B
from paper_2508_02124_amd.paged_cache import CacheRows, PagedCache
from paper_2508_02124_amd.torch_api import DynamicMaskAttention

H_Q, H_KV, D, N = 4, 2, 64, 3


class Recorded(PagedCache):
    """A cache whose buffers live on the CPU and whose calls are written down instead of launched."""

    def __init__(self):
        self.shape = B.make_cache_shape(2, 8, 4, 16, H_Q, H_KV, D)
        self.device, self.dtype, self.calls = torch.device("cpu"), torch.bfloat16, []
        self.pages = torch.zeros(B.dma_cache_bytes(self.shape), dtype=torch.uint8)
        self.seq_lens, self.block_table = self._ints(2), self._ints(2, 4)
        self.free_list = self._ints(12)

    def _call_with(self, shape, entry, *args):
        self.calls.append((entry.__name__, shape, args))


def module(cross_head, **more):
    torch.manual_seed(0)
    return DynamicMaskAttention(**{**dict(num_heads=H_Q, num_kv_heads=H_KV, head_dim=D, keep_window=8, cross_head=cross_head), **more})


def rows(n=N):
    ints = lambda m: torch.zeros(m, dtype=torch.int32)
    return CacheRows(ints(3), ints(n), ints(n), ints(n), ints(2))


def values(heads, d=D, n=N, dtype=torch.bfloat16, device="cpu"):
    return torch.zeros((n, heads, d), dtype=dtype, device=device)


@pytest.mark.parametrize("cross_head", [False, True])
def test_bad_arguments_launch_nothing(cross_head):
    good = dict(q=values(H_Q), k=values(H_KV), v=values(H_KV))
    bad = [(ValueError, dict(v=values(H_KV - 1))), (ValueError, dict(v=values(H_KV, D // 2))), (ValueError, dict(v=values(H_KV, n=N - 1))),
           (ValueError, dict(v=values(H_KV, n=N + 1))), (ValueError, dict(v=values(H_KV)[:, 0])),
           (TypeError, dict(v=values(H_KV, dtype=torch.float32))), (RuntimeError, dict(v=values(H_KV, device="meta"))),
           (ValueError, dict(k=values(H_KV - 1))), (TypeError, dict(k=values(H_KV, dtype=torch.float16))),
           (RuntimeError, dict(k=values(H_KV, device="meta")))]
    for error, more in bad:
        cache = Recorded()
        with pytest.raises(error):
            module(cross_head).step(**{**good, **more}, cache=cache, rows=rows())
        assert cache.calls == [], more
    for error, m in ((TypeError, module(cross_head).bfloat16()), (RuntimeError, module(cross_head, device="meta")),
                     (ValueError, module(cross_head, num_heads=H_Q + 2)), (ValueError, module(cross_head, head_dim=128)),
                     (ValueError, module(cross_head, num_heads=8, num_kv_heads=4))):
        cache = Recorded()
        with pytest.raises(error):
            m.step(**good, cache=cache, rows=rows())
        assert cache.calls == []


def test_calls_of_a_step():
    for cross_head, names in ((False, ["dma_cache_append", "dma_cache_decode"]),
                              (True, ["dma_scores_xhead", "dma_cache_append", "dma_cache_decode"])):
        cache = Recorded()
        o = module(cross_head).step(values(H_Q), values(H_KV), values(H_KV), cache, rows())
        assert [c[0] for c in cache.calls] == names and o.shape == (N, H_Q, D)


@pytest.mark.parametrize("form", ["contiguous", "odd place", "part of a projection", "transposed"])
def test_values_of_the_cross_head_scores(form):
    """dma_scores_xhead reads whole rows at addresses of 16 bytes: the values as they are, or a copy of them."""
    n = 5
    v = torch.randn(n, H_KV, D).bfloat16()
    given = {"contiguous": lambda: v, "odd place": lambda: torch.cat((v.new_zeros(1), v.flatten()))[1:].view(v.shape),
             "part of a projection": lambda: torch.cat((v, v, v), 1)[:, H_KV:2 * H_KV],
             "transposed": lambda: v.transpose(0, 1).contiguous().transpose(0, 1)}[form]()
    cache = Recorded()
    module(True).step(values(H_Q, n=n), v, given, cache, rows(n))
    _, shape, (V, W, A, z) = cache.calls[0]
    assert (shape.T, shape.H_q, shape.H_kv, shape.d) == (n, H_Q, H_KV, D)
    assert V.is_contiguous() and V.data_ptr() % 16 == 0 and torch.equal(V, v) and z.shape == (H_Q, n)


@pytest.mark.parametrize("cross_head", [False, True])
def test_what_decode_refuses_is_refused_before_the_rows_go_in(cross_head):
    """A step whose attention cannot run leaves the cache as it was."""
    good = dict(q=values(H_Q), k=values(H_KV), v=values(H_KV), rows=rows())
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    bad = [(ValueError, dict(q=values(H_Q - 1))), (ValueError, dict(q=values(H_Q, n=N + 1))), (TypeError, dict(q=values(H_Q, dtype=torch.float32))),
           (RuntimeError, dict(q=values(H_Q, device="meta"))), (ValueError, dict(rows=rows()._replace(row_len=ints(N + 1)))),
           (TypeError, dict(rows=rows()._replace(row_req=ints(N).long()))), (B.DmaError, dict(max_len=-1))]
    for error, more in bad:
        cache = Recorded()
        with pytest.raises(error):
            module(cross_head).step(**{**good, **more}, cache=cache)
        assert cache.calls == [], more
    for more in (dict(keep_window=0), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan"))):
        cache = Recorded()
        with pytest.raises(B.DmaError) as e:
            module(cross_head, **more).step(**good, cache=cache)
        assert cache.calls == [] and e.value.status == B.DMA_EINVAL


def test_rows_and_window_of_a_step():
    """The limit of dma_cache_decode, (n_rows + 8) * H_q * ceil(window / 256) < 2^22, at both its sides."""
    cache, window, n = Recorded(), 1 << 21, 120
    cache.shape = B.make_cache_shape(2, 8, 1 << 18, 16, H_Q, H_KV, D)
    assert (n + 8) * H_Q * (window // 256) == 1 << 22
    assert B.dma_cache_decode_bytes(cache.shape, n, window) == 0 < B.dma_cache_decode_bytes(cache.shape, n - 1, window)
    with pytest.raises(B.DmaError) as e:
        module(False, keep_window=window).step(values(H_Q, n=n), values(H_KV, n=n), values(H_KV, n=n), cache, rows(n))
    assert cache.calls == [] and e.value.status == B.DMA_EUNSUPPORTED
    cache._check_decode(values(H_Q, n=n - 1), window, rows(n - 1), 0.0, 0)


@pytest.mark.parametrize("page_size", [0, -16, 24])
def test_page_sizes_are_refused_by_the_library(page_size):
    for max_tokens in (None, 50):
        with pytest.raises(B.DmaError):
            PagedCache(2, 4, H_Q, H_KV, D, page_size=page_size, max_tokens=max_tokens)
