"""Rotary positions and prefixes through PagedCache, DynamicMaskAttention and rotary: what is refused, before any launch (on the CPU, with the
launches recorded)."""
import pytest
import torch

from paper_2508_02124_amd import binding as B
from paper_2508_02124_amd.paged_cache import CachePrefixes
from paper_2508_02124_amd.torch_api import DynamicMaskAttention, rotary, rotary_freqs
from test_paged_cache_refusals import D, H_KV, H_Q, N, Recorded, module, rows, values


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def shared(n=2, **more):
    return CachePrefixes(ints(n), ints(n), ints(2))._replace(**more)


FREQS = rotary_freqs(D)


def test_calls_of_a_step():
    for cross_head in (False, True):
        for dim, prefixes in ((D, None), (16, shared()), (0, shared())):
            cache = Recorded()
            o = module(cross_head, rotary_dim=dim).step(values(H_Q), values(H_KV), values(H_KV), cache, rows(), prefixes=prefixes)
            names = [c[0] for c in cache.calls]
            assert names == ["dma_scores_xhead"] * cross_head + ["dma_cache_append_rope" if dim else "dma_cache_append",
                                                                 "dma_cache_decode_prefix" if prefixes else "dma_cache_decode"]
            assert o.shape == (N, H_Q, D)
            if dim:
                args = cache.calls[-2][2]
                assert args[16].numel() == dim // 2 and args[17] == dim and args[13] == (2 if prefixes else 0)


@pytest.mark.parametrize("cross_head", [False, True])
def test_a_step_is_refused_before_the_rows_go_in(cross_head):
    good = dict(q=values(H_Q), k=values(H_KV), v=values(H_KV), rows=rows(), prefixes=shared())
    bad = [(ValueError, dict(prefixes=shared(len=ints(3)))), (TypeError, dict(prefixes=shared(req=ints(2).long()))),
           (ValueError, dict(prefixes=shared(of=ints(3)))), (RuntimeError, dict(prefixes=shared(of=ints(2).to("meta")))),
           (B.DmaError, dict(max_prefix=-1)), (ValueError, dict(q=values(H_Q + 1))), (TypeError, dict(q=values(H_Q, dtype=torch.float32))),
           (ValueError, dict(rows=rows()._replace(row_len=ints(N + 1)))), (B.DmaError, dict(prefixes=shared(4097))),
           (ValueError, dict(v=values(H_KV - 1))), (TypeError, dict(k=values(H_KV, dtype=torch.float16)))]
    for error, more in bad:
        cache = Recorded()
        with pytest.raises(error):
            module(cross_head, rotary_dim=32).step(**{**good, **more}, cache=cache)
        assert cache.calls == [], more
    cache = Recorded()
    with pytest.raises(TypeError):
        module(cross_head, rotary_dim=32).bfloat16().step(**good, cache=cache)
    assert cache.calls == []


@pytest.mark.parametrize("error,more", [(ValueError, dict(freqs=FREQS[:4])), (ValueError, dict(freqs=torch.zeros(D))), (TypeError, dict(freqs=FREQS.double())),
                                        (ValueError, dict(freqs=FREQS[None])), (ValueError, dict(freqs=FREQS[:0])), (ValueError, dict(freqs=rotary_freqs(2 * D)[::2][:32])),
                                        (ValueError, dict(q=values(H_Q - 1))), (ValueError, dict(W=None)), (ValueError, dict(z=torch.zeros(H_Q, N))),
                                        (TypeError, dict(W=torch.zeros(H_Q, D, dtype=torch.bfloat16))), (ValueError, dict(prefixes=shared(len=ints(1)))),
                                        (ValueError, dict(rows=rows()._replace(row_req=ints(N - 1)))), (ValueError, dict(v=values(H_KV, n=N + 1)))])
def test_append_rotary(error, more):
    good = dict(rows=rows(), q=values(H_Q), k=values(H_KV), v=values(H_KV), freqs=FREQS, W=torch.zeros(H_Q, D), A=torch.zeros(H_Q), prefixes=shared())
    cache = Recorded()
    assert cache.append_rotary(**good).shape == (N, H_Q, D) and cache.append_rotary(**{**good, "q": None}) is None and len(cache.calls) == 2
    cache = Recorded()
    with pytest.raises(error):
        cache.append_rotary(**{**good, **more})
    assert cache.calls == []


def test_prefixes():
    cache = Recorded()
    cache.seq_lens = torch.tensor([5, 9], dtype=torch.int32)
    p = cache.prefixes([1], [0, -1])
    assert p.req.tolist() == [1] and p.len.tolist() == [9] and p.of.tolist() == [0, -1] and p.len.dtype == torch.int32
    assert cache.prefixes([1, 0], [0, 1], [3, 4]).len.tolist() == [3, 4]
    for error, call in ((ValueError, lambda: cache.prefixes([1], [0])), (ValueError, lambda: cache.prefixes([1], [0, 0], [1, 2])),
                        (TypeError, lambda: cache.prefixes(torch.zeros(1, dtype=torch.int64), [0, 0], [1]))):
        with pytest.raises(error):
            call()


def test_rotary_arguments():
    q, k = torch.zeros(4, 2, 64), torch.zeros(4, 1, 64)
    with pytest.raises(RuntimeError):
        rotary(q, k, rotary_freqs(64), positions=ints(4))           # no CPU path
    for dim in (8, 24, 80, -16):
        with pytest.raises(ValueError):
            DynamicMaskAttention(2, 1, 64, 8, rotary_dim=dim)
    m = DynamicMaskAttention(2, 1, 64, 8, rotary_dim=32, rotary_base=100.0)
    assert m.rotary_freqs.dtype == torch.float32 and torch.equal(m.rotary_freqs, (100.0 ** (-torch.arange(16, dtype=torch.float64) / 16)).float())
    assert set(m.state_dict()) == {"W", "A"} == set(DynamicMaskAttention(2, 1, 64, 8).state_dict())
    with pytest.raises(ValueError):
        DynamicMaskAttention(2, 1, 64, 8)(q, k, k, cu_seqlens=ints(2), positions=ints(4))


def test_a_module_s_frequencies_are_not_rounded():
    m = DynamicMaskAttention(H_Q, H_KV, D, 8, rotary_dim=32, rotary_base=5e5)
    want = m.rotary_freqs.clone()
    assert want.dtype == torch.float32 and torch.equal(want, (5e5 ** (-torch.arange(0, 32, 2).double() / 32)).float())
    for there in (lambda: m.bfloat16(), lambda: m.float(), lambda: m.double()):
        assert torch.equal(there().rotary_freqs, want) and m.rotary_freqs.dtype == torch.float32
    empty = DynamicMaskAttention(H_Q, H_KV, D, 8, rotary_dim=32, rotary_base=5e5, device="meta")
    assert empty.rotary_freqs.device.type == "meta" and torch.equal(empty.to_empty(device="cpu").rotary_freqs, want)
    assert "rotary_freqs" not in m.state_dict()
