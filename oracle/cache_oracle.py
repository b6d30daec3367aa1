"""CPU oracle of the paged 4-bit cache: plain loops over the definitions, values in fp64.

TEST INFRASTRUCTURE ONLY, like dma_oracle; it shares no code with the HIP path.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
SERVED, NO_PAGES, TOO_LONG, NO_ROWS = 0, 1, 2, 3


class Pages:
    """The requests' pages, the free ones and the lengths, as plain Python lists."""

    def __init__(self, n_reqs, n_pages, max_pages, page_size):
        self.max_pages, self.ps = max_pages, page_size
        self.lens = [0] * n_reqs
        self.tables = [[] for _ in range(n_reqs)]
        self.free = list(range(n_pages - 1, -1, -1))     # a stack: the last one is taken first

    def assign(self, change, n_rows):
        """(cu_rows, row_req, row_len, slots, status) of one step."""
        ps = self.ps
        for b, c in enumerate(change):
            if c < 0:
                self.lens[b] = max(0, self.lens[b] + c)
                keep = -(-self.lens[b] // ps)
                self.free += self.tables[b][keep:]
                self.tables[b] = self.tables[b][:keep]
        have, asked, row = len(self.free), 0, 0
        cu, status = [0], []
        req, length, slots = [-1] * n_rows, [0] * n_rows, [-1] * n_rows
        for b, c in enumerate(change):
            grow, state = max(0, c), SERVED
            first, row = row, row + grow
            if grow:
                need = -(-(self.lens[b] + grow) // ps) - len(self.tables[b])
                if len(self.tables[b]) + need > self.max_pages:
                    state = TOO_LONG
                elif row > n_rows:
                    state = NO_ROWS
                else:
                    asked += need
                    if need and asked > have:
                        state = NO_PAGES
                if state == SERVED:
                    for _ in range(need):
                        self.tables[b].append(self.free.pop())
                    for i in range(grow):
                        pos = self.lens[b] + i
                        req[first + i], length[first + i] = b, pos + 1
                        slots[first + i] = self.tables[b][pos // ps] * ps + pos % ps
                    self.lens[b] += grow
            cu.append(min(row, n_rows))
            status.append(state)
        return cu, req, length, slots, status

    def table(self):
        out = np.full((len(self.tables), self.max_pages), -1, np.int32)
        for b, t in enumerate(self.tables):
            out[b, : len(t)] = t
        return out


def quantise(x):
    """What the cache holds of x [..., d] (float64 values of fp32 or bf16 inputs): the nearest code value of every block of 32
    channels, ties to the even code; NaN for a block that is not finite."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(-1, 32)
    out = np.empty_like(blocks)
    for i, v in enumerate(blocks):
        top = np.abs(v).max()
        if not np.isfinite(v).all():
            out[i] = np.nan
            continue
        e = -125
        if top > 0:
            mantissa, exponent = np.frexp(top)           # top = 2 mantissa * 2^(exponent - 1)
            e = exponent - 3 + (1 if 2 * mantissa >= 1.75 else 0)
        step = 2.0 ** min(max(e, -125), 125)
        a = np.abs(v) / step
        gap = np.abs(a[:, None] - GRID)
        near = gap == gap.min(1, keepdims=True)
        code = np.array([max(np.flatnonzero(n), key=lambda c: c % 2 == 0) for n in near])
        out[i] = np.copysign(GRID[code], v) * step
    return out.reshape(x.shape)


def decode_row(q, K, V, z, k, scale):
    """One row: q [H_q, d], its n keys K, V [n, H_kv, d], z [H_q, n].  (o, lse, positions kept per head)."""
    H_q, d = q.shape
    n, H_kv = K.shape[0], K.shape[1]
    o, lse, kept = np.zeros((H_q, d)), np.full(H_q, -np.inf), []
    for h in range(H_q):
        zh = z[h].astype(np.float64) + 0.0
        best = np.sort(np.argsort(-zh, kind="stable")[: min(k, n)])
        kept.append(best)
        use = best[~np.isneginf(zh[best])]
        if len(use) == 0:
            continue
        g = h // (H_q // H_kv)
        s = K[use, g] @ q[h] * scale + zh[use]
        m = s.max()
        p = np.exp(s - m)
        o[h] = p @ V[use, g] / p.sum()
        lse[h] = m + np.log(p.sum())
    return o, lse, kept
