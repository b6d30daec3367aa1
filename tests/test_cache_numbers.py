"""Numbers that do not fit the 32 bits of the paged cache's entry points, without a GPU: refused, or, where a larger one means the same as the
largest that counts, taken as that one; never cut to their lowest bits."""
import os

import pytest

from paper_2508_02124_amd import binding as B
from paper_2508_02124_amd.paged_cache import PagedCache
from test_cache import P, shape
from test_paged_cache_refusals import D, H_KV, H_Q, N, Recorded, module, rows, values


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g
        g.build()


@pytest.mark.parametrize("x", [1 << 31, (1 << 32) + 4, 1 << 40, -(1 << 31) - 1, 4 - (1 << 32)])
def test_numbers_beyond_32_bits_are_refused_not_cut(x):
    s = shape()
    for name in ("n_reqs", "n_pages", "max_pages", "page_size", "H_q", "H_kv", "d", "dtype", "max_len"):
        with pytest.raises(OverflowError):
            shape(**{name: x})
    for call in (lambda: B.dma_cache_decode_bytes(s, x, 5), lambda: B.dma_cache_decode_bytes(s, 4, x),
                 lambda: B.dma_cache_assign(s, x, *[P] * 9, stream=0),
                 lambda: B.dma_cache_append(s, x, P, 256, P, 256, P, P, None, P, P, stream=0),
                 lambda: B.dma_cache_read(s, x, P, P, P, P, P, stream=0),
                 lambda: B.dma_cache_decode(s, x, 9, 0.0, P, 1024, *[P] * 8, 1 << 60, stream=0),
                 lambda: B.dma_cache_decode(s, 0, x, 0.0, P, 1024, *[P] * 8, 1 << 60, stream=0)):
        with pytest.raises(OverflowError):
            call()


@pytest.mark.parametrize("window", [64, 65, 1 << 31, (1 << 32) + 3, 1 << 40])
def test_windows_beyond_the_longest_request_keep_all(window):
    cache = Recorded()                               # (4 pages of 16 tokens a request)
    o, lse, kept = cache.decode(values(H_Q), window, rows())
    (name, _, args), = cache.calls
    assert name == "dma_cache_decode" and args[:2] == (N, 64) and kept.shape == (N, H_Q, 64)
    cache = Recorded()
    module(False, keep_window=window).step(values(H_Q), values(H_KV), values(H_KV), cache, rows())
    assert cache.calls[-1][2][:2] == (N, 64)


@pytest.mark.parametrize("max_len,want", [(0, 0), (1, 1), (64, 64), (65, 64), (1 << 31, 64), ((1 << 32) + 1, 64)])
def test_bounds_beyond_the_longest_request_are_none(max_len, want):
    for call in (lambda c: c.decode(values(H_Q), 8, rows(), max_len=max_len),
                 lambda c: module(False).step(values(H_Q), values(H_KV), values(H_KV), c, rows(), max_len=max_len)):
        cache = Recorded()
        call(cache)
        assert cache.calls[-1][1].max_len == want


def test_sizes_of_the_object():
    for more in (dict(n_reqs=(1 << 32) + 2), dict(n_pages=(1 << 32) + 2), dict(max_tokens=1 << 50)):
        with pytest.raises(OverflowError):
            PagedCache(**{**dict(n_reqs=2, n_pages=4, num_heads=H_Q, num_kv_heads=H_KV, head_dim=D), **more})
