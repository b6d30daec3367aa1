"""PagedCache.prefixes: a prefix whose holder is not there has no tokens, whether its length is given or not, so that rows are turned to the
positions that the decode sees (on the CPU, with the launches recorded)."""
import pytest
import torch

from test_paged_cache_refusals import D, H_KV, H_Q, Recorded, module, rows, values

REQ = [1, 2, -1, 0, 2 ** 31 - 1, -2 ** 31]
LENGTH = [7, 50, 50, 3, 1, 9]


@pytest.mark.parametrize("form", ["sequences", "tensors"])
def test_a_given_length_of_a_holder_that_is_not_there(form):
    cache = Recorded()
    cache.seq_lens = torch.tensor([5, 9], dtype=torch.int32)
    ints = (lambda x: torch.tensor(x, dtype=torch.int32)) if form == "tensors" else list
    given = ints(LENGTH)
    p = cache.prefixes(ints(REQ), ints([0, 1]), given)
    assert p.len.tolist() == [7, 0, 0, 3, 0, 0] and p.len.dtype == torch.int32 and p.req.tolist() == REQ
    assert list(given) == LENGTH or given.tolist() == LENGTH                       # (the caller's own stays as it is)
    assert cache.prefixes(ints(REQ), ints([0, 1])).len.tolist() == [9, 0, 0, 5, 0, 0]
    module(False, rotary_dim=D).step(values(H_Q), values(H_KV), values(H_KV), cache, rows(), prefixes=p)
    append, decode = cache.calls
    assert append[0] == "dma_cache_append_rope" and append[2][14] is p.len and decode[0] == "dma_cache_decode_prefix" and decode[2][12] is p.len


def test_refusals_stay():
    cache = Recorded()
    cache.seq_lens = torch.tensor([5, 9], dtype=torch.int32)
    long = lambda x: torch.tensor(x)
    for error, call in ((ValueError, lambda: cache.prefixes([1, 0], [0, 0], [4])), (ValueError, lambda: cache.prefixes([1], [0, 0], [4, 4])),
                        (TypeError, lambda: cache.prefixes([1], [0, 0], long([4]))), (TypeError, lambda: cache.prefixes(long([1]), [0, 0], [4])),
                        (TypeError, lambda: cache.prefixes(long([1]), [0, 0])),
                        (RuntimeError, lambda: cache.prefixes([1], [0, 0], long([4]).to("meta").int()))):
        with pytest.raises(error):
            call()
