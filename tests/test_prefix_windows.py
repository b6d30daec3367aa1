"""Windows beyond the longest request, behind a prefix: a row sees the tokens of two requests (on the CPU, with the launches recorded)."""
import pytest

from paper_2508_02124_amd import binding as B
from test_paged_cache_refusals import H_KV, H_Q, N, Recorded, module, rows, values
from test_rotary_objects_refusals import shared

LONGEST = 64     # tokens of a request of Recorded


@pytest.mark.parametrize("window", [1, 8, 63, 64, 65, 100, 127, 128, 129, 5000, 2 ** 40])
def test_a_window_reaches_over_a_prefix_and_the_own_keys(window):
    cache = Recorded()
    cache.decode_prefix(values(H_Q), window, rows(), shared())
    cache.decode(values(H_Q), window, rows())
    module(False, keep_window=window).step(values(H_Q), values(H_KV), values(H_KV), cache, rows(), prefixes=shared())
    got = [(name, args[1]) for name, _, args in cache.calls if "decode" in name]
    assert got == [("dma_cache_decode_prefix", min(window, 2 * LONGEST)), ("dma_cache_decode", min(window, LONGEST)),
                   ("dma_cache_decode_prefix", min(window, 2 * LONGEST))]


def test_the_longest_windows_stay_numbers_of_32_bits_and_the_limit_on_rows_is_the_same():
    cache = Recorded()
    cache.shape = B.make_cache_shape(2, 8, 1 << 22, 256, H_Q, H_KV, 64)          # requests of up to 2^30 tokens
    with pytest.raises(B.DmaError) as e:                                         # (more than 2^22 parts of 256 keys)
        cache.decode_prefix(values(H_Q), 2 ** 40, rows(), shared())
    assert e.value.status == B.DMA_EUNSUPPORTED and cache.calls == []
    cache.shape = B.make_cache_shape(2, 8, 1 << 17, 256, 1, 1, 64)               # 2^25: (n + 8) * 2^17 < 2^22 for up to 23 rows and prefixes
    for n, taken in ((21, True), (22, False)):
        call = lambda: cache.decode_prefix(values(1, n=n), 2 ** 40, (rows(n).row_req, rows(n).row_len), shared())
        if taken:
            call()
            assert cache.calls[-1][2][1] == 2 ** 26
        else:
            with pytest.raises(B.DmaError):
                call()
    assert len(cache.calls) == 1 and N < 21
