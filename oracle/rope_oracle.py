"""CPU oracle of the rotary positions: the definition in extended precision (angles of far positions in more than 64 bits).

TEST INFRASTRUCTURE ONLY, like dma_oracle; it shares no code with the HIP path.
"""
from __future__ import annotations

import numpy as np


def document_positions(cu):
    """The place of every token in its document."""
    return np.concatenate([np.arange(b - a) for a, b in zip(cu[:-1], cu[1:])] or [np.zeros(0, int)])


def angles(positions, freqs):
    """[T, rot / 2]: position (an integer) times freqs (the exact values of fp32 numbers)."""
    return np.asarray(positions, np.longdouble)[:, None] * np.asarray(freqs, np.float32).astype(np.longdouble)


def rotate(x, positions, freqs, interleaved=False, inverse=False):
    """x [T, H, d] turned, and the bound of one value's size that its rounding errors scale with, |x1| + |x2| of its pair (0 where
    nothing turns)."""
    a = angles(positions, freqs)
    cos, sin = np.cos(a).astype(np.float64)[:, None], np.sin(a).astype(np.float64)[:, None]
    sin = -sin if inverse else sin
    x = np.asarray(x, np.float64)
    half = a.shape[1]
    i = np.arange(half)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out, size = x.copy(), np.zeros_like(x)
    x1, x2 = x[..., first], x[..., second]
    out[..., first] = x1 * cos - x2 * sin
    out[..., second] = x1 * sin + x2 * cos
    size[..., first] = size[..., second] = np.abs(x1) + np.abs(x2)
    return out, size
