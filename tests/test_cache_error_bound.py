"""How far the values that the paged cache holds are from those given, over all magnitudes of fp32, by the oracle's definition."""
import numpy as np
import pytest

from oracle import cache_oracle as co

LOW, HIGH = 5 * 2.0 ** -127, 1.75 * 2.0 ** 127   # largest values from which on, and up to which, a fifth of it holds


def blocks(low, high, seed, n=3000):
    """Blocks of 32 whose largest magnitude is anywhere between low and high, the others around it, as fp32."""
    r = np.random.default_rng(seed)
    top = np.exp2(r.uniform(np.log2(low), np.log2(high), (n, 1)))
    x = r.uniform(-1, 1, (n, 32)) * top
    x[:, :1] = np.where(r.random((n, 1)) < 0.5, top, -top)
    x = np.clip(x, -float(np.finfo(np.float32).max), float(np.finfo(np.float32).max)).astype(np.float32).astype(np.float64)
    amax = np.abs(x).max(1, keepdims=True)
    inside = ((amax >= low) & (amax < high))[:, 0]
    return x[inside], amax[inside]


def worst(low, high, seed):
    x, top = blocks(low, high, seed)
    assert len(x) > 1000
    return np.abs(co.quantise(x) - x), top


@pytest.mark.parametrize("low,high", [(LOW, 2.0 ** -120), (2.0 ** -124, 2.0 ** 124), (2.0 ** 122, HIGH)])
def test_a_fifth_of_the_largest(low, high):
    error, top = worst(low, high, 1)
    assert (error <= top / 5).all() and (error > 0.19 * top).any()


def test_small_blocks():
    """The power of two is at least 2^-125: codes are 2^-126 apart there, and half of that is the most."""
    error, top = worst(2.0 ** -149, LOW, 2)
    assert (error <= 2.0 ** -127).all() and (error > 0.9 * top).any()
    assert co.quantise(np.full(32, 2.0 ** -127))[0] == 0 and co.quantise(np.full(32, 2.0 ** -126))[0] == 2.0 ** -126


def test_large_blocks():
    """The power of two is at most 2^125: values end at 6 * 2^125."""
    x, top = blocks(HIGH, 2.0 ** 128, 3)
    held = co.quantise(x)
    assert (np.abs(held) <= 6 * 2.0 ** 125).all()
    assert (np.abs(held - x) <= top / 4).all() and (np.abs(held - x) > 0.24 * top).any()
