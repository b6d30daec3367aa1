"""dma_cache_decode_prefix with more (row, head) or (prefix, head) pairs than the selection's scratch has room for at once (8192), against
the oracle on rows from every share."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from cache_harness import normal
from paper_2508_02124_amd import binding as B
from paper_2508_02124_amd.paged_cache import PagedCache
from paper_2508_02124_amd.torch_api import DynamicMaskAttention
from test_gpu_cache_prefix import Shared, ints

pytestmark = pytest.mark.gpu

HELD = 3        # requests that hold prefixes, and as many with long rows of their own; behind them requests of a few tokens
SHORT = 40


class Many(Shared):
    """n_prefixes prefixes, all of them beginnings of what the first requests hold; rows of long requests, and of short ones that are
    behind prefixes from the first to the last."""

    def __init__(self, dev, held, own, n_prefixes, ps, H_q, dtype="bf16", z="ordinary"):
        rng = np.random.default_rng(n_prefixes)
        lens = [*own, *(1 + i % 9 for i in range(SHORT))]
        super().__init__(dev, held, lens, [-1] * len(lens), ps, H_q, 1, 64, dtype, z, seed=3)
        holders = rng.integers(0, HELD, n_prefixes)
        length = [int(rng.integers(held[b] // 2, held[b] + 1)) for b in holders]
        of = [-1] * HELD + [int(rng.integers(0, n_prefixes)) for _ in own] + [int(x) for x in np.linspace(0, n_prefixes - 1, SHORT)]
        self.prefix_req, self.prefix_len, self.req_prefix, self.n_pre = ints(dev, list(holders)), ints(dev, length), ints(dev, of), n_prefixes

    def rows(self, n_rows, rng):
        """Rows of the long requests at places from the first to the last, some of the short ones between them."""
        rows = [(HELD + i % 3, int(rng.integers(self.lens[i % 3] // 2, self.lens[i % 3] + 1))) for i in range(n_rows)]
        for i, r in enumerate(np.linspace(0, n_rows - 1, SHORT).astype(int)):
            if i % 2 or n_rows == SHORT:
                rows[r] = (2 * HELD + i, self.lens[3 + i])
        return rows


# held, own, prefixes, rows, window, page size, bounds on own keys and on prefixes: launches of the selection
CASES = {
    "rows, short": ((3000, 700, 50), (5000, 4000, 2100), 1, 300, 512, 64, 0, 0),
    "prefixes, short": ((600, 500, 400), (20, 30, 40), 300, SHORT, 200, 16, 0, 0),
    "both, short": ((3000, 2500, 2900), (3500, 2200, 3400), 270, 270, 900, 32, 0, 0),
    "rows, long; prefixes, short": ((4000, 700, 50), (13000, 12600, 14000), 2, 300, 600, 64, 0, 4000),
    "prefixes, long; rows, short": ((13000, 12500, 14000), (2500, 2400, 700), 300, 90, 600, 64, 2500, 0),
    "both, long, three and two": ((13000, 12400, 13500), (13100, 12700, 700), 600, 300, 700, 16, 0, 0),
}


@pytest.mark.parametrize("kind", ["ordinary", "equal"])
@pytest.mark.parametrize("name", CASES)
def test_rows_of_every_share(gpu, name, kind):
    print(f"[case] prefix shares {name} {kind}", flush=True)
    held, own, n_prefixes, n_rows, k, ps, max_len, max_prefix = CASES[name]
    s = Many(gpu, held, own, n_prefixes, ps, 32, z=kind)
    s.cache.shape.max_len = max_len
    rng = np.random.default_rng(1)
    rows = s.rows(n_rows, rng)
    q = normal(gpu, 5, n_rows, 32, 64).to(s.cache.type)
    req, length = ints(gpu, [b for b, _ in rows]), ints(gpu, [n for _, n in rows])
    o, lse = s.decode(q, k, req, length, max_prefix=max_prefix)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    some = sorted({0, 1, n_rows // 3, n_rows // 2, n_rows // 2 + 1, 2 * n_rows // 3 + 1, n_rows - 2, n_rows - 1} | {r for r in (149, 150, 255, 256) if r < n_rows})
    if len(held) * max(held) > 30000:
        some = some[::2] + some[-1:]                 # (what the oracle's loops take)
    at = torch.tensor(some, device=gpu)
    s.check(q[at], k, [rows[i] for i in some], (o[at], lse[:, at]))
    # a call of these rows alone makes fewer lists: the same kept sets, sums in other parts
    alone = s.decode(q[at], k, req[at], length[at], max_prefix=max_prefix)
    assert torch.allclose(alone[1], lse[:, at], atol=1e-5, rtol=0)


def test_captured_call_of_several_launches(gpu):
    """Three launches of prefixes beside two of rows over the same scratch, in a graph: every replay is the eager call."""
    held, own, n_prefixes, n_rows, k, ps, _, _ = CASES["both, long, three and two"]
    s = Many(gpu, held, own, n_prefixes, ps, 32)
    rows = s.rows(n_rows, np.random.default_rng(2))
    q = normal(gpu, 5, n_rows, 32, 64).to(s.cache.type)
    req, length = ints(gpu, [b for b, _ in rows]), ints(gpu, [n for _, n in rows])
    c = s.cache
    size = B.dma_cache_decode_prefix_bytes(c.shape, n_rows, k, n_prefixes, 0)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=gpu)
    o, lse = torch.zeros((n_rows, 32, 64), dtype=c.type, device=gpu), torch.zeros((32, n_rows), device=gpu)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.dma_cache_decode_prefix(c.shape, n_rows, k, 0.0, q, q.stride(0), c.pages, c.table, req, length, n_prefixes, 0, s.prefix_req,
                                  s.prefix_len, s.req_prefix, o, lse, ws, size)
    for i in range(3):
        q.mul_(0.9)
        length.sub_((length > 20).int() * i)
        ref = s.decode(q, k, req, length)
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, ref[0]) and torch.equal(lse, ref[1])


@pytest.mark.parametrize("P,m,window,max_tokens", [(3000, 1500, 512, 8192), (14000, 2600, 700, 16640), (900, 2300, 2100, 2400)])
def test_a_long_question_behind_a_prefix(gpu, P, m, window, max_tokens):
    """A prompt's thousands of rows go in and attend in one step behind a shared prefix, turned to their positions: the answers of the same
    tokens as one request, for every row, with bounds on the lengths and without."""
    H_q, H_kv, d = 32, 4, 64
    torch.manual_seed(1)
    layer = DynamicMaskAttention(H_q, H_kv, d, window, device=gpu, rotary_dim=d)
    make = lambda longest: PagedCache(3, 2 * (P + m) // 64 + 8, H_q, H_kv, d, page_size=64, max_tokens=longest, device=gpu)
    split = lambda x: x.split((H_q, H_kv, H_kv), 1)
    first, rest = normal(gpu, 1, P, H_q + 2 * H_kv, d, dtype=torch.bfloat16), normal(gpu, 2, m, H_q + 2 * H_kv, d, dtype=torch.bfloat16)
    one = make(P + m + 64)
    for x, n in ((first, P), (rest, m)):
        ref_rows = one.assign([0, n, 0])
        ref = layer.step(*split(x), one, ref_rows).float()
    for bounds in (dict(), dict(max_len=m, max_prefix=P)):
        two = make(max_tokens)
        layer.step(*split(first), two, two.assign([0, 0, P]))
        shared, rows = two.prefixes([2], [-1, 0, -1]), two.assign([0, m, 0])
        got = layer.step(*split(rest), two, rows, prefixes=shared, **bounds).float()
        for a, b in zip(one.read(ref_rows.slots), two.read(rows.slots)):
            assert torch.equal(a, b)
        # the same number but for weights off by 2^-16 and one rounding each (2^-8 of it, twice)
        assert ((got - ref).abs() <= 2.0 ** -7 * ref.abs() + 2.0 ** -13).all()
