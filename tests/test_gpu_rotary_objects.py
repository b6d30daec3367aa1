"""Rotary positions and shared prefixes as training and serving programs use them: gradients of a turned layer, whole runs over the cache."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from cache_harness import f64, normal
from oracle import cache_oracle as co, rope_oracle as ro
from paper_2508_02124_amd import binding as B
from paper_2508_02124_amd.paged_cache import PagedCache
from paper_2508_02124_amd.torch_api import DynamicMaskAttention, rotary, rotary_freqs
from test_gpu_rope import bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_are_turned_back(gpu, dtype, interleaved):
    """Against the formula (the transpose), from gradients that are expanded, transposed or parts of others."""
    T, H_q, H_kv, d, name = 37, 4, 2, 64, "bf16" if dtype == torch.bfloat16 else "f32"
    freqs, cu = rotary_freqs(48, 100.0, gpu), torch.tensor([0, 20, 20, T], dtype=torch.int32, device=gpu)
    positions = ro.document_positions(cu.tolist())
    fused = normal(gpu, 1, T, H_q + H_kv, d, dtype=dtype).requires_grad_()
    Q, K = fused.split((H_q, H_kv), 1)
    Qo, Ko = rotary(Q, K, freqs, cu, interleaved=interleaved)
    w = normal(gpu, 2, H_q, T, d, dtype=dtype).transpose(0, 1)
    (g,) = torch.autograd.grad((Qo * w).sum() + Ko.sum(), fused)
    both = np.concatenate((f64(w), np.ones((T, H_kv, d))), 1)
    ref, size = ro.rotate(both, positions, freqs.cpu().numpy(), interleaved, True)
    assert (np.abs(f64(g) - ref) <= bound(ref, size, name)).all()
    # the same by given positions, of which one is enough for both
    again = rotary(Q, K, freqs, positions=torch.from_numpy(positions.astype(np.int32)).to(gpu), interleaved=interleaved)
    assert torch.equal(again[0], Qo) and torch.equal(again[1], Ko)


def test_gradients_against_differences(gpu):
    """(f(x + e v) - f(x - e v)) / 2 e with f = sum w y^2 / 2, summed in 64 bits: exact for a quadratic f but for the roundings of y, of
    x +- e v and of g.  A value of y is off by 3 u (|x1| + |x2|), which changes its term by at most |w y| times that; with |w y| <= 20 and
    |x1| + |x2| <= 12 (5 standard deviations) the three together stay below n * 30 * 12 * 3 u / e."""
    T, H, d, e = 18, 2, 64, 0.25
    freqs, pos = rotary_freqs(64, 50.0, gpu), torch.arange(T, device=gpu).int() * 1000
    x, v, w = (normal(gpu, i, T, H, d) for i in (1, 2, 3))
    k = normal(gpu, 4, T, 1, d)
    f = lambda y: (w.double() * rotary(y, k, freqs, positions=pos)[0].double().square()).sum() / 2
    x.requires_grad_()
    (g,) = torch.autograd.grad(f(x), x)
    want = (f(x.detach() + e * v) - f(x.detach() - e * v)) / (2 * e)
    got = (g.double() * v.double()).sum()
    assert abs(float(want - got)) <= T * H * d * 30 * 12 * 3 * 2.0 ** -24 / e


def test_second_derivatives(gpu):
    T, d = 5, 64
    freqs, pos = rotary_freqs(64, device=gpu), torch.arange(T, device=gpu).int() + 9
    x, k = normal(gpu, 1, T, 2, d).requires_grad_(), normal(gpu, 2, T, 1, d)
    y = rotary(x, k, freqs, positions=pos)[0]
    (g,) = torch.autograd.grad((y ** 3).sum() / 6, x, create_graph=True)       # R^T (y^2 / 2)
    v = normal(gpu, 3, T, 2, d)
    (h,) = torch.autograd.grad((g * v).sum(), x)                               # R^T (y * R v)
    turn = lambda a, inverse=False: ro.rotate(a, pos.cpu().numpy(), freqs.cpu().numpy(), inverse=inverse)[0]
    ref = turn(turn(f64(x)) * turn(f64(v)), True)
    # three turns, each off by 3 u of |x1| + |x2| < 10 times factors below 10
    assert np.abs(f64(h) - ref).max() <= 3 * 3 * 2.0 ** -24 * 10 * 10 * 2


def test_refusals(gpu):
    q, k, f, cu = torch.zeros(4, 2, 64, device=gpu), torch.zeros(4, 1, 64, device=gpu), rotary_freqs(64, device=gpu), torch.tensor([0, 4], device=gpu).int()
    for error, call in ((ValueError, lambda: rotary(q, k, f)), (ValueError, lambda: rotary(q, k, f, cu, cu)), (ValueError, lambda: rotary(q, k[:3], f, cu)),
                        (ValueError, lambda: rotary(q, k, f, positions=cu)), (TypeError, lambda: rotary(q, k.bfloat16(), f, cu)),
                        (TypeError, lambda: rotary(q, k, f.double(), cu)), (TypeError, lambda: rotary(q, k, f, cu.long())),
                        (TypeError, lambda: rotary(q.half(), k.half(), f, cu)), (B.DmaError, lambda: rotary(q, k, f[:4], cu)),
                        (B.DmaError, lambda: rotary(q, k, rotary_freqs(80, device=gpu), cu)), (RuntimeError, lambda: rotary(q, k, f.cpu(), cu))):
        with pytest.raises(error):
            call()


def test_module_turns_before_it_attends(gpu):
    """A module with rotary_dim is rotary followed by the same module without, values and gradients, batched and packed."""
    torch.manual_seed(3)
    m = DynamicMaskAttention(4, 2, 64, 24, device=gpu, rotary_dim=32, rotary_base=500.0)
    plain = DynamicMaskAttention(4, 2, 64, 24, device=gpu)
    plain.load_state_dict(m.state_dict())
    qkv = normal(gpu, 1, 2, 50, 8, 64, dtype=torch.float32).requires_grad_()
    q, k, v = qkv.split((4, 2, 2), 2)
    o = m(q, k, v)
    flat = [x.reshape(100, *x.shape[2:]) for x in (q, k, v)]
    cu = torch.tensor([0, 50, 100], dtype=torch.int32, device=gpu)
    tq, tk = rotary(flat[0], flat[1], m.rotary_freqs, cu)
    ref = plain(tq, tk, flat[2], cu)
    packed = m(*flat, cu)
    given = m(q, k, v, positions=torch.arange(50, device=gpu).int().expand(2, 50))
    assert torch.equal(o.reshape(ref.shape), ref) and torch.equal(packed, ref) and torch.equal(given, o)
    w = normal(gpu, 2, 100, 4, 64)
    g0 = torch.autograd.grad((ref * w).sum(), (qkv, plain.W, plain.A), retain_graph=True)
    g1 = torch.autograd.grad((o.reshape(ref.shape) * w).sum(), (qkv, m.W, m.A))
    for a, b in zip(g0, g1):   # (the backward's atomics: last bits)
        assert torch.allclose(a, b, rtol=1e-5, atol=1e-5 * float(a.abs().max()))


class Server:
    """Requests behind prefixes, beside the same tokens as plain lists in 64 bits: what the cache should hold and answer."""

    def __init__(self, gpu, dtype, cross_head, rotary_dim, interleaved, window):
        self.H_q, self.H_kv, self.d, self.dtype = 4, 2, 64, dtype
        self.m = DynamicMaskAttention(4, 2, 64, window, device=gpu, cross_head=cross_head, rotary_dim=rotary_dim, rotary_base=100.0,
                                      rotary_interleaved=interleaved)
        self.cache = PagedCache(8, 80, 4, 2, 64, page_size=16, max_tokens=480, dtype=dtype, device=gpu)
        self.tokens = {}          # request -> (K, V as they came, z)
        self.gpu, self.seed = gpu, 0

    def values(self, n):
        self.seed += 1
        return normal(self.gpu, self.seed, n, 8, 64, dtype=self.dtype).split((4, 2, 2), 1)

    def scores(self, v):
        W, A = f64(self.m.W), f64(self.m.A)
        v = f64(v)
        x = np.stack([(v.reshape(len(v), -1) if W.shape[1] > 64 else v[:, h // 2]) @ W[h] for h in range(4)])
        return np.exp(A[:, None] * np.logaddexp(0.0, x))

    def grow(self, change, n_rows, prefixes=None, of=()):
        rows = self.cache.assign(change, n_rows)
        q, k, v = self.values(n_rows)
        o = self.m.step(q, k, v, self.cache, rows, prefixes=prefixes)
        for r, (b, slot) in enumerate(zip(rows.row_req.tolist(), rows.slots.tolist())):
            if b >= 0:
                have = self.tokens.setdefault(b, [])
                have.append((f64(k)[r], f64(v)[r], slot))
        for b, c in enumerate(change):
            if c < 0:
                self.tokens[b] = self.tokens.get(b, [])[:max(0, len(self.tokens.get(b, [])) + c)]
        return rows, q, o

    def check(self, rows, q, o, of):
        """The outputs against the oracle over a row's prefix and own tokens; the bound of test_gpu_cache.check_rows with the terms of
        test_gpu_cache_prefix, and for the turned queries (rounded to their type: half a step of q, a factor e^(2 E_q) on a weight)."""
        half, u, freqs = torch.finfo(self.dtype).eps / 2, 2.0 ** -24, self.m.rotary_freqs
        k = self.m.keep_window
        held = {b: [x.double().cpu().numpy() for x in self.cache.read(torch.tensor([t[2] for t in ts], dtype=torch.int32, device=self.gpu))]
                for b, ts in self.tokens.items() if ts}
        for r, (b, n) in enumerate(zip(rows.row_req.tolist(), rows.row_len.tolist())):
            if b < 0:
                assert (o[r] == 0).all()
                continue
            p = of[b] if b < len(of) else -1
            parts = ([held[p]] if p >= 0 else []) + [[held[b][0][:n], held[b][1][:n], held[b][2][:, :n]]]
            K, V, z = (np.concatenate(x, axis) for x, axis in zip(zip(*parts), (0, 0, 1)))
            position = n - 1 + (len(self.tokens[p]) if p >= 0 else 0)
            qr = f64(q)[r][None]
            if freqs is not None:
                qr, _ = ro.rotate(qr, [position], freqs.cpu().numpy(), self.m.rotary_interleaved)
            ro_, rl, rk = co.decode_row(qr[0], K, V, z, k, self.d ** -0.5)
            for h in range(4):
                g, use = h // 2, rk[h]
                pw = np.exp(K[use, g] @ qr[0, h] / math.sqrt(self.d) + z[h, use] - rl[h])
                size = (np.abs(K[use, g]) @ np.abs(qr[0, h]) / math.sqrt(self.d)).max()
                E = (self.d + 4) * u * (size + np.abs(z[h, use]).max()) + (half + 3 * 2 * u) * (size if freqs is not None else 0.0)
                w = np.expm1(2 * E) + 2.0 ** -20 + 2.0 ** -16 + (len(use) + 16) * u
                lim = w * (pw @ np.abs(V[use, g])) + half * np.abs(ro_[h]) * (1 + w)
                assert (np.abs(f64(o)[r, h] - ro_[h]) <= lim).all(), (r, h)

    def check_cache(self, of):
        """What the cache holds of every token: the codes of K turned to its place, of V as it is, and the scores."""
        for b, ts in self.tokens.items():
            if not ts:
                continue
            K, V, z = self.cache.read(torch.tensor([t[2] for t in ts], dtype=torch.int32, device=self.gpu))
            p = of[b] if b < len(of) else -1
            at = np.arange(len(ts)) + (len(self.tokens[p]) if p >= 0 else 0)
            ref = np.stack([t[0] for t in ts])
            if self.m.rotary_freqs is not None:
                ref, _ = ro.rotate(ref, at, self.m.rotary_freqs.cpu().numpy(), self.m.rotary_interleaved)
            assert (f64(K) == co.quantise(ref)).all() and (f64(V) == co.quantise(np.stack([t[1] for t in ts]))).all()
            want = self.scores(torch.from_numpy(np.stack([t[1] for t in ts])))
            assert (np.abs(f64(z) - want) <= 1e-5 * np.abs(want)).all()


@pytest.mark.parametrize("dtype,cross_head,rotary_dim,interleaved,window", [
    (torch.bfloat16, False, 64, False, 40), (torch.float32, False, 32, True, 100), (torch.bfloat16, True, 64, False, 1000), (torch.float32, True, 0, False, 30)])
def test_a_server_with_prefixes(gpu, dtype, cross_head, rotary_dim, interleaved, window):
    """Prefixes go in, requests start behind them, take steps of one and several tokens, lose drafts and end; every answer against the
    oracle, and the cache's contents at the end."""
    s = Server(gpu, dtype, cross_head, rotary_dim, interleaved, window)
    of = [6, 6, 7, -1, 6, 7, -1, -1]                                       # requests 6 and 7 hold the prefixes
    check = lambda got: s.check(*got, of)
    check(s.grow([0, 0, 0, 0, 0, 0, 200, 53], 253))
    shared = s.cache.prefixes([6, 7], [{6: 0, 7: 1}.get(p, -1) for p in of])
    check(s.grow([3, 17, 30, 40, 0, 1, 0, 0], 100, shared))                # (rows behind the last one)
    for step in range(4):
        check(s.grow([1, 1, 4, 1, step, 1, 0, 0], 12, shared))
        s.grow([0, 0, -3, 0, 0, -2 ** 31 if step == 2 else 0, 0, 0], 0, shared)
    s.check_cache(of)
    free = int(s.cache.free_list[0])
    s.cache.assign([-2 ** 31] * 8, 0)                                      # all pages come back once
    assert int(s.cache.free_list[0]) == 80 > free


def test_a_shared_prefix_is_a_longer_request(gpu):
    """The same tokens once behind a prefix and once as one request: the cache holds the same, and the answers agree."""
    torch.manual_seed(1)
    m = DynamicMaskAttention(4, 2, 64, 60, device=gpu, rotary_dim=64)
    one, two = (PagedCache(4, 40, 4, 2, 64, page_size=16, device=gpu) for _ in range(2))
    q, k, v = normal(gpu, 1, 130, 8, 64, dtype=torch.bfloat16).split((4, 2, 2), 1)
    rows = one.assign([130, 0, 0, 0])
    ref = m.step(q, k, v, one, rows)
    first = two.assign([0, 0, 100, 0])
    m.step(q[:100], k[:100], v[:100], two, first)
    shared = two.prefixes([2], [-1, 0, -1, -1])
    rest = two.assign([0, 30, 0, 0])
    got = m.step(q[100:], k[100:], v[100:], two, rest, prefixes=shared)
    for a, b in zip(one.read(rows.slots[100:]), two.read(rest.slots)):
        assert torch.equal(a, b)
    # both outputs are the same number but for weights off by 2^-16 and one rounding each
    assert ((got.float() - ref[100:].float()).abs() <= 2.0 ** -7 * ref[100:].float().abs() + 2.0 ** -13).all()


def test_captured_step_replays(gpu):
    """assign, append with rotation and decode behind a prefix in one graph: every replay is the eager step."""
    torch.manual_seed(2)
    m = DynamicMaskAttention(4, 2, 128, 50, device=gpu, rotary_dim=128)

    def run(captured):
        cache = PagedCache(6, 60, 4, 2, 128, page_size=16, device=gpu)
        seed = lambda i, n: normal(gpu, i, n, 8, 128, dtype=torch.bfloat16)
        fused = seed(0, 90)
        m.step(*fused.split((4, 2, 2), 1), cache, cache.assign([0, 0, 0, 0, 0, 90], 90))
        shared = cache.prefixes([5], [0, 0, 0, -1, 0, -1])
        change = torch.zeros(6, dtype=torch.int32, device=gpu)
        buf = seed(1, 10)
        out = torch.zeros((10, 4, 128), dtype=torch.bfloat16, device=gpu)

        def step():
            out.copy_(m.step(*buf.split((4, 2, 2), 1), cache, cache.assign(change, 10), prefixes=shared))

        graph = torch.cuda.CUDAGraph()
        if captured:
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step()
        outs = []
        for i, c in enumerate(([5, 1, 0, 2, 1, 0], [1, 1, 1, 1, 1, 0], [1, 0, 4, 1, 1, 0], [-3, 1, 1, 1, 1, 0], [1, 1, 1, 1, 1, 0])):
            change.copy_(torch.tensor(c, dtype=torch.int32))
            buf.copy_(seed(10 + i, 10))
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            outs.append(out.clone())
        return outs

    for a, b in zip(run(True), run(False)):
        assert torch.equal(a, b)


def test_prefixes_held_by_requests_that_are_not_there(gpu):
    cache = PagedCache(3, 8, 2, 1, 64, page_size=16, device=gpu)
    cache.assign([0, 9, 20], 29)
    shared = cache.prefixes([2, 3, -1, 1, 2 ** 31 - 1], [0, 1, 2])
    assert shared.len.tolist() == [20, 0, 0, 9, 0] and shared.len.dtype == torch.int32
    assert cache.prefixes([], [-1] * 3).len.shape == (0,)
    with pytest.raises(ValueError):
        cache.prefixes([2], [0, 0])
    with pytest.raises(ValueError):
        cache.prefixes([2, 1], [0, 0, 0], [4])


def test_frequencies_get_no_gradient(gpu):
    q, f = torch.zeros(4, 2, 64, device=gpu), rotary_freqs(64, device=gpu).requires_grad_()
    with pytest.raises(ValueError):
        rotary(q, q, f, positions=torch.arange(4, device=gpu).int())


def test_a_captured_backward(gpu):
    """Forward and backward in one graph; every replay against the eager result."""
    freqs, pos = rotary_freqs(64, 100.0, gpu), torch.arange(30, device=gpu).int()
    x = normal(gpu, 1, 30, 3, 64).requires_grad_()
    w = normal(gpu, 2, 30, 2, 64)
    def run():
        y, _ = rotary(x[:, :2], x[:, 2:], freqs, positions=pos)
        (g,) = torch.autograd.grad(y, x, w)
        return y.detach(), g
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, g = run()
    for seed in (3, 4, 5):
        with torch.no_grad():
            x.copy_(normal(gpu, seed, 30, 3, 64))
        pos.add_(11)
        graph.replay()
        torch.cuda.synchronize()
        ye, ge = run()
        assert torch.equal(y, ye) and torch.equal(g, ge)
