"""The paged cache without a GPU: the oracle's definitions, sizes and layouts, and what the entry points refuse before any launch."""
import os

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2508_02124_amd import binding as B

P = 0x1000   # an aligned dummy address: never dereferenced by a call that is refused


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return B.lib()


def shape(**more):
    args = dict(n_reqs=4, n_pages=10, max_pages=5, page_size=16, H_q=8, H_kv=2, d=128)
    args.update(more)
    return B.make_cache_shape(**args)


def test_values_of_the_oracle():
    x = np.zeros(64)
    x[:8] = [6, -5, 5.01, 2.5, 0.25, 0.75, -0.26, 1.25]              # amax 6: step 1
    x[32:35] = [7.0, 3.5, -6.9]                                       # mantissa 1.75: step 2
    q = co.quantise(x)
    assert q[:8].tolist() == [6, -4, 6, 2, 0, 1, -0.5, 1]
    assert q[32:35].tolist() == [8, 4, -6]                            # 7 / 2 = 3.5 -> 4, 1.75 -> 2, 3.45 -> 3
    x[40] = np.inf
    assert np.isnan(co.quantise(x)[32:]).all() and (co.quantise(x)[:32] == q[:32]).all()
    r = np.random.default_rng(1).standard_normal((50, 32)) * np.exp(np.random.default_rng(2).uniform(-60, 60, (50, 1)))
    top = np.abs(r).max(1, keepdims=True)
    assert (np.abs(co.quantise(r) - r) <= top / 5 * (1 + 1e-12)).all()   # the largest is 3.5 to 7 steps: at most 1 of 5, 1 - 4 / 5 below that


def test_pages_of_the_oracle():
    p = co.Pages(3, 5, 3, 16)
    cu, req, length, slots, status = p.assign([17, 1, 0], 20)
    assert cu == [0, 17, 18, 18] and status == [0, 0, 0] and p.tables == [[0, 1], [2], []]
    assert slots[15:18] == [15, 16, 32] and length[15:18] == [16, 17, 1] and req[17:] == [1, -1, -1]
    _, _, _, slots, status = p.assign([32, 1, 33], 99)                   # too long, in its page, too few pages left
    assert status == [2, 0, 1] and slots[32:34] == [33, -1] and p.lens == [17, 2, 0]
    _, _, _, _, status = p.assign([-1, -2**31, 2], 1)                    # pages come back first; rows behind the capacity
    assert status == [0, 0, 3] and p.lens == [16, 0, 0] and p.free == [4, 3, 1, 2]


@pytest.mark.parametrize("H_q,H_kv,d,ps", [(8, 2, 128, 16), (1, 1, 64, 16), (3, 3, 256, 256), (32, 8, 128, 64)])
def test_layout(H_q, H_kv, d, ps):
    s = shape(H_q=H_q, H_kv=H_kv, d=d, page_size=ps)
    l = B.dma_cache_describe(s)
    assert l.off_codes == 0 and l.off_scales == H_kv * ps * d and l.off_scores == l.off_scales + H_kv * ps * d // 16
    used = l.off_scores + 4 * H_q * ps
    assert l.page_bytes % 256 == 0 and used <= l.page_bytes < used + 256
    assert B.dma_cache_bytes(s) == 10 * l.page_bytes and B.dma_cache_free_bytes(s) == 4 * (10 + 4)
    assert B.dma_cache_decode_bytes(s, 3, 100) >= 0 and B.dma_cache_decode_bytes(s, 0, 100) == 0


EINVAL = [dict(n_reqs=0), dict(n_pages=0), dict(max_pages=0), dict(H_q=0), dict(H_kv=0), dict(H_q=9), dict(n_reqs=-1), dict(max_len=-1)]
UNSUPPORTED = [dict(d=96), dict(d=32), dict(dtype=2), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=0),
               dict(n_reqs=4097), dict(n_pages=(1 << 26) + 1), dict(max_pages=(1 << 26) + 1), dict(H_q=514, H_kv=2), dict(H_q=8192, H_kv=4096)]


def refused(status, call, *args):
    with pytest.raises(B.DmaError) as e:
        call(*args, stream=0)
    assert e.value.status == status, args


@pytest.mark.parametrize("more", EINVAL + UNSUPPORTED)
def test_shapes_refused(more):
    s, status = shape(**more), B.DMA_EINVAL if more in EINVAL else B.DMA_EUNSUPPORTED
    assert B.dma_cache_bytes(s) == B.dma_cache_free_bytes(s) == B.dma_cache_decode_bytes(s, 1, 1) == 0
    refused(status, B.dma_cache_reset, s, P, P, P)
    refused(status, B.dma_cache_assign, s, 4, *[P] * 9)
    refused(status, B.dma_cache_append, s, 4, P, 4096, P, 4096, P, P, P, P, P)
    refused(status, B.dma_cache_read, s, 4, P, P, P, P, P)
    refused(status, B.dma_cache_decode, s, 4, 9, 0.0, P, 1 << 20, *[P] * 8, 1 << 30)
    with pytest.raises(B.DmaError) as e:
        B.dma_cache_describe(s)
    assert e.value.status == status


def test_arguments_refused():
    s, inval = shape(), B.DMA_EINVAL
    for i in range(3):
        refused(inval, B.dma_cache_reset, s, *[None if j == i else P for j in range(3)])
    for i in range(9):
        refused(inval, B.dma_cache_assign, s, 4, *[None if j == i else P for j in range(9)])
    refused(inval, B.dma_cache_assign, s, -1, *[P] * 9)
    row = 2 * 128
    good = [4, P, row, P, row, P, P, None, P, P]
    for at, bad in ((0, -1), (1, None), (1, P + 8), (2, row - 8), (2, row + 4), (2, -row), (3, None), (3, P + 2), (4, 0),
                    (4, row + 1), (5, P + 4), (6, None), (8, None), (9, None), (9, P + 8)):
        refused(inval, B.dma_cache_append, s, *[bad if i == at else x for i, x in enumerate(good)])
    refused(inval, B.dma_cache_append, s, 4, P, row, P, row, None, P, None, P, P)      # neither W nor z
    good = [4, P, P, P, P, P]
    for at, bad in ((0, -1), (1, None), (2, None), (2, P + 8), (3, None), (3, P + 8), (4, None), (4, P + 8), (5, None)):
        refused(inval, B.dma_cache_read, s, *[bad if i == at else x for i, x in enumerate(good)])
    need = B.dma_cache_decode_bytes(shape(max_pages=100), 4, 1000)
    big, row = shape(max_pages=100), 8 * 128
    good = [4, 1000, 0.0, P, row, P, P, P, P, P, P, P, P, need]
    for at, bad in ((0, -1), (1, 0), (1, -5), (2, -1.0), (2, float("nan")), (3, None), (3, P + 8), (4, row - 8), (4, row + 4),
                    (5, None), (5, P + 4), (6, None), (8, None), (9, None), (9, P + 8), (10, None), (11, None), (11, P + 4), (12, P + 4)):
        refused(inval, B.dma_cache_decode, big, *[bad if i == at else x for i, x in enumerate(good)])
    for at, bad in ((12, None), (13, need - 1)):
        refused(B.DMA_EWORKSPACE, B.dma_cache_decode, big, *[bad if i == at else x for i, x in enumerate(good)])
    refused(inval, B.dma_cache_decode, s, 5, 9, 0.0, P, row, P, P, None, *[P] * 5, 1 << 30)   # row r is request r: only four
    refused(B.DMA_EUNSUPPORTED, B.dma_cache_decode, big, 1 << 17, 1000, 0.0, P, row, *[P] * 8, 1 << 40)
    assert B.dma_cache_decode_bytes(big, 1 << 17, 1000) == 0 and B.dma_cache_decode_bytes(big, 4, 0) == 0


def test_numbers_of_rows_refused():
    s, many = shape(), (1 << 28) + 1
    refused(B.DMA_EUNSUPPORTED, B.dma_cache_assign, s, many, *[P] * 9)
    refused(B.DMA_EUNSUPPORTED, B.dma_cache_append, s, many, P, 256, P, 256, P, P, None, P, P)
    refused(B.DMA_EUNSUPPORTED, B.dma_cache_read, s, many, P, P, P, P, P)
    refused(B.DMA_EUNSUPPORTED, B.dma_cache_decode, s, many, 9, 0.0, P, 1024, *[P] * 8, 1 << 60)
    assert B.dma_cache_bytes(shape(n_pages=1 << 26)) > 0 and B.dma_cache_free_bytes(shape(max_pages=1 << 26)) > 0


def test_no_rows_is_no_work():
    """Nothing is enqueued (no GPU is here), and the row arrays may be missing."""
    s = shape()
    B.dma_cache_append(s, 0, None, 256, None, 256, None, None, None, None, None, stream=0)
    B.dma_cache_read(s, 0, None, None, None, None, None, stream=0)
    B.dma_cache_decode(s, 0, 5, 0.0, None, 1024, *[None] * 8, 0, stream=0)
