"""dma_rope on the GPU against the definition in extended precision.

Error of one value, with u = 2^-24: cosine and sine are rounded to fp32 (u / 2 of at most 1 each, since the angles' own error is far
below), one product is rounded (u of it) and then their sum (u of it): at most (|x1| + |x2|) * 2.5 u, written with 3 u for the terms in
u^2.  bf16 results have one more rounding, 2^-8 of the value.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import rope_oracle as ro
from paper_2508_02124_amd import binding as B
from cache_harness import f64, normal

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, B.DMA_BF16), "f32": (torch.float32, B.DMA_F32)}


def bound(ref, size, dtype):
    off = size * 3 * 2.0 ** -24
    return off + (2.0 ** -8 * (np.abs(ref) + off) if dtype == "bf16" else 0.0)


def frequencies(dev, rot, base=10000.0):
    i = torch.arange(rot // 2, dtype=torch.float64)
    return (base ** (-2.0 * i / rot)).float().to(dev)


def check(got, x, positions, freqs, dtype, interleaved, inverse):
    ref, size = ro.rotate(f64(x), positions, freqs.cpu().numpy(), interleaved, inverse)
    err = np.abs(f64(got) - ref)
    assert np.isfinite(err).all() and (err <= bound(ref, size, dtype)).all(), float((err - bound(ref, size, dtype)).max())


CASES = [  # lengths, H_q, H_kv, d, rot
    ((1,), 32, 8, 128, 128), ((5, 0, 3, 1), 4, 2, 64, 64), ((70, 131), 3, 1, 128, 32), ((33,), 5, 5, 256, 256), ((9, 8), 2, 1, 256, 48),
    ((1000,), 8, 2, 64, 16), ((3, 2, 0, 0, 4), 7, 7, 128, 112)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward_and_back(gpu, case, interleaved, dtype):
    lengths, H_q, H_kv, d, rot = CASES[case]
    T, real = sum(lengths), TYPES[dtype][0]
    cu = np.concatenate(([0], np.cumsum(lengths))).astype(np.int32)
    shape = B.make_shape(T, len(lengths), H_q, H_kv, d, 1, dtype=TYPES[dtype][1])
    freqs = frequencies(gpu, rot)
    qkv = normal(gpu, case, T, H_q + 2 * H_kv, d, dtype=real)      # parts of one projection's output
    Q, K = qkv[:, :H_q], qkv[:, H_q:H_q + H_kv]
    cu_t = torch.from_numpy(cu).to(gpu)
    for inverse in (False, True):
        Qo, Ko = (torch.full(x.shape, float("nan"), dtype=real, device=gpu) for x in (Q, K))
        B.dma_rope(shape, Q, Q.stride(0), K, K.stride(0), cu_t, None, freqs, rot, interleaved, inverse, Qo, Qo.stride(0), Ko, Ko.stride(0))
        for x, y in ((Q, Qo), (K, Ko)):
            check(y, x, ro.document_positions(cu), freqs, dtype, interleaved, inverse)
            assert torch.equal(x[..., rot:], y[..., rot:])
    # out into a projection's gradient: what lies between the rows stays
    out = torch.full_like(qkv, 7.0)
    Qc, Kc = Q.contiguous(), K.contiguous()
    B.dma_rope(shape, Qc, H_q * d, Kc, H_kv * d, cu_t, None, freqs, rot, interleaved, True, out, out.stride(0), out[:, H_q:], out.stride(0))
    assert torch.equal(out[:, :H_q], Qo) and torch.equal(out[:, H_q:H_q + H_kv], Ko) and (out[:, H_q + H_kv:] == 7).all()
    # one of the two alone; in place
    Q2, K2 = Qc.clone(), Kc.clone()
    B.dma_rope(shape, Q2, H_q * d, None, 0, cu_t, None, freqs, rot, interleaved, True, Q2, H_q * d, None, 0)
    B.dma_rope(shape, None, 0, K2, H_kv * d, cu_t, None, freqs, rot, interleaved, True, None, 0, K2, H_kv * d)
    assert torch.equal(Q2, Qo) and torch.equal(K2, Ko)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(gpu, dtype):
    T, H, d, rot = 41, 2, 128, 128
    real = TYPES[dtype][0]
    rng = np.random.default_rng(3)
    positions = np.concatenate(([0, -1, 2 ** 31 - 1, -(2 ** 31), 2 ** 30, 131071], rng.integers(-(2 ** 31), 2 ** 31, T - 6))).astype(np.int32)
    freqs = frequencies(gpu, rot, 500000.0)
    freqs[1] = 1.0 + 2.0 ** -23     # (an angle of 55 bits)
    x = normal(gpu, 5, T, H, d, dtype=real)
    y = torch.empty_like(x)
    shape = B.make_shape(T, 1, H, H, d, 1, dtype=TYPES[dtype][1])
    B.dma_rope(shape, x, H * d, None, 0, None, torch.from_numpy(positions).to(gpu), freqs, rot, False, False, y, H * d, None, 0)
    check(y, x, positions, freqs, dtype, False, False)


def test_documents_by_the_thousand(gpu):
    """The search for a token's document, with empty ones at the borders of its steps."""
    rng = np.random.default_rng(1)
    lengths = rng.integers(0, 4, 5000)
    lengths[:200] = 0
    lengths[-100:] = 0
    cu = np.concatenate(([0], np.cumsum(lengths))).astype(np.int32)
    T = int(cu[-1])
    x = normal(gpu, 8, T, 1, 64)
    y = torch.empty_like(x)
    freqs = frequencies(gpu, 64)
    B.dma_rope(B.make_shape(T, len(lengths), 1, 1, 64, 1, dtype=B.DMA_F32), x, 64, None, 0, torch.from_numpy(cu).to(gpu), None, freqs, 64, True,
               False, y, 64, None, 0)
    check(y, x, ro.document_positions(cu), freqs, "f32", True, False)


def test_channels_that_stay_keep_their_bits_and_pairs_their_infinities(gpu):
    x = normal(gpu, 2, 6, 1, 64)
    x[0, 0, 20], x[1, 0, 40], x[2, 0, 3] = float("inf"), float("nan"), float("inf")
    y = torch.empty_like(x)
    B.dma_rope(B.make_shape(6, 1, 1, 1, 64, 1, dtype=B.DMA_F32), x, 64, None, 0, None, torch.arange(6, device=gpu).int(), frequencies(gpu, 16), 16,
               False, False, y, 64, None, 0)
    assert torch.equal(y[..., 16:].view(torch.int32), x[..., 16:].view(torch.int32))
    off = ~torch.isfinite(y[..., :16])
    assert off.nonzero().tolist() == [[2, 0, 3], [2, 0, 11]]


def test_other_stream_and_graph(gpu):
    T, H, d = 200, 4, 128
    shape, freqs = B.make_shape(T, 1, H, H, d, 1), frequencies(gpu, d)
    cu = torch.tensor([0, T], dtype=torch.int32, device=gpu)
    x = normal(gpu, 4, T, H, d, dtype=torch.bfloat16)
    ref, y = torch.empty_like(x), torch.zeros_like(x)
    call = lambda out, stream=None: B.dma_rope(shape, x, H * d, None, 0, cu, None, freqs, d, False, False, out, H * d, None, 0, stream)
    call(ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(y, side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(y)
    for seed in range(3):
        x.copy_(normal(gpu, 10 + seed, T, H, d, dtype=torch.bfloat16))
        call(ref)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref)


def test_more_tokens_than_a_launch_takes(gpu):
    """2^22 + 37 tokens: the last ones are turned, to their own positions, and nothing behind them is written."""
    T, d = (1 << 22) + 37, 64
    x = normal(gpu, 1, 1024, 1, d, dtype=torch.bfloat16).repeat(T // 1024 + 1, 1, 1)[:T]
    y = torch.full((T + 5, 1, d), 3.0, dtype=torch.bfloat16, device=gpu)
    freqs, cu = frequencies(gpu, d, 500000.0), torch.tensor([0, 1 << 22, T], dtype=torch.int32, device=gpu)
    B.dma_rope(B.make_shape(T, 2, 1, 1, d, 1), x, d, None, 0, cu, None, freqs, d, False, False, y, d, None, 0)
    at = torch.cat((torch.arange(0, 1 << 22, 99991), torch.arange((1 << 22) - 9, T))).to(gpu)
    positions = torch.where(at < 1 << 22, at, at - (1 << 22)).cpu().numpy()
    check(y[at], x[at], positions, freqs, "bf16", False, False)
    assert (y[T:] == 3).all()
