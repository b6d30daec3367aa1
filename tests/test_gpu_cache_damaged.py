"""dma_cache_assign over lists that hold page numbers out of range: the rows of such pages are not there, all others are as usual."""
from __future__ import annotations

import pytest
import torch

from cache_harness import GpuCache, normal

pytestmark = pytest.mark.gpu


# 40 rows are written by the first launch, 5000 by the second.  Of pages of 16 tokens the numbers 2^28 and 2^28 + 3 shifted by 4 bits are 0 and 48
# again, the place of another request's token.
@pytest.mark.parametrize("n_rows", [40, 5000])
@pytest.mark.parametrize("bad", [1 << 28, (1 << 28) + 3, 12, -1, 2**31 - 1, -2**31])
def test_pages_out_of_range_are_rows_that_are_not_there(gpu, n_rows, bad):
    cache = GpuCache(gpu, 3, 12, 6, 16, 2, 1, 64)
    first = cache.assign([20, 20, 0], 40)
    k = normal(gpu, 1, 40, 1, 64).to(cache.type)
    cache.append(k, k, first[3], z=normal(gpu, 2, 2, 40))
    before = cache.pages.clone()
    # the free pages, from the top of the stack: 4, 5, 6, ...; request 0 takes two (the second one's entry is damaged), request 1 stays in its
    # last page, whose entry in the table is, request 2 takes the next one of the stack
    assert cache.free[0] == 8 and cache.free[4 + 5:4 + 8].tolist() == [6, 5, 4]
    cache.free[4 + 6] = bad
    cache.table[1, 1] = bad
    cu, req, length, slots, status = (x.tolist() for x in cache.assign([40, 3, 10], n_rows))
    want = [(0, 21 + i, (1 * 16 + 4 + i) if i < 12 else (4 * 16 + i - 12)) for i in range(28)] + [(-1, 0, -1)] * 12 + [(-1, 0, -1)] * 3
    if n_rows > 53:
        want += [(2, i + 1, 6 * 16 + i) for i in range(10)]
        assert status == [0, 0, 0] and cu == [0, 40, 43, 53]
    else:                                            # (the rows of requests 1 and 2 end behind the last one)
        want = want[:40]
        assert status == [0, 3, 3] and cu == [0, 40, 40, 40]
    want += [(-1, 0, -1)] * (n_rows - len(want))
    assert list(zip(req, length, slots)) == want
    # nothing of the tokens that were there changes
    n = sum(c >= 0 for c in slots)
    x = normal(gpu, 3, n_rows, 1, 64).to(cache.type)
    cache.append(x, x, torch.tensor(slots, dtype=torch.int32, device=gpu), z=normal(gpu, 4, 2, n_rows))
    old = first[3]
    now = cache.read(old)
    cache.pages, after = before, cache.pages
    assert all(torch.equal(a, b) for a, b in zip(now, cache.read(old)))
    assert n == sum(a >= 0 for _, _, a in want) and not torch.equal(after, before)


def test_a_last_page_out_of_range_in_the_first_launch(gpu):
    cache = GpuCache(gpu, 2, 12, 6, 16, 2, 1, 64)
    cache.assign([20, 5], 25)
    cache.table[0, 1] = 1 << 28
    cu, req, length, slots, status = (x.tolist() for x in cache.assign([3, 2], 5))
    assert (req, length, slots) == ([-1, -1, -1, 1, 1], [0, 0, 0, 6, 7], [-1, -1, -1, 2 * 16 + 5, 2 * 16 + 6]) and status == [0, 0]
