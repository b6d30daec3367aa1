"""dma_cache_decode_prefix: what is refused, before any launch (so without a GPU), and the sizes of its scratch."""
import pytest

from paper_2508_02124_amd import binding as B

P = 0x1000


def call(n=4, reqs=4, k=8, **more):
    a = dict(H_q=4, q=P, qs=256, pages=P, table=P, req=P, length=P, np=2, mp=0, pr=P, pl=P, of=P, o=P, lse=P, ws=P, size=1 << 40, scale=0.0, max_pages=8,
             n_pages=8)
    a.update(more)
    shape = B.make_cache_shape(reqs, a["n_pages"], a["max_pages"], 16, a["H_q"], 2, 64)
    return lambda: B.dma_cache_decode_prefix(shape, n, k, a["scale"], a["q"], a["qs"], a["pages"], a["table"], a["req"], a["length"], a["np"], a["mp"],
                                             a["pr"], a["pl"], a["of"], a["o"], a["lse"], a["ws"], a["size"], stream=0)


def status(f):
    with pytest.raises(B.DmaError) as e:
        f()
    return e.value.status


@pytest.mark.parametrize("more", [dict(n=-1), dict(k=0), dict(np=-1), dict(mp=-1), dict(q=None), dict(pages=None), dict(table=None), dict(length=None),
                                  dict(pr=None), dict(pl=None), dict(of=None), dict(o=None), dict(lse=None), dict(q=P + 2), dict(pages=P + 8),
                                  dict(o=P + 8), dict(ws=P + 8), dict(qs=248), dict(qs=260), dict(scale=-1.0), dict(scale=float("nan")),
                                  dict(n=5, req=None), dict(H_q=3)])
def test_arguments(more):
    assert status(call(**more)) == B.DMA_EINVAL


def test_sizes():
    assert status(call(np=4097)) == B.DMA_EUNSUPPORTED
    assert status(call(ws=None)) == B.DMA_EWORKSPACE
    shape = B.make_cache_shape(4, 8, 8, 16, 4, 2, 64)
    need = B.dma_cache_decode_prefix_bytes(shape, 4, 8, 2)
    assert need > 0 and status(call(size=need - 1)) == B.DMA_EWORKSPACE
    assert B.dma_cache_decode_prefix_bytes(shape, 0, 8, 2) == 0
    call(n=0, q=None, pages=None, table=None, length=None, o=None, lse=None, ws=None, size=0)()
    for bad in ((-1, 8, 2, 0), (4, 0, 2, 0), (4, 8, -2, 0), (4, 8, 4097, 0), (4, 8, 2, -3)):
        assert B.dma_cache_decode_prefix_bytes(shape, *bad) == 0
    # the limit of dma_cache_decode, prefixes counted as rows
    wide = B.make_cache_shape(4096, 1 << 18, 1 << 18, 16, 4, 2, 64)
    window = 1 << 21                                     # (n + 8) * 4 * 8192 < 2^22
    assert B.dma_cache_decode_prefix_bytes(wide, 100, window, 20) == 0 < B.dma_cache_decode_prefix_bytes(wide, 100, window, 19)
    with pytest.raises(OverflowError):
        call(np=1 << 32)()


def test_more_rows_and_prefixes_never_need_less():
    for max_len in (0, 500):
        shape = B.make_cache_shape(64, 4096, 1024, 64, 32, 8, 128, max_len=max_len)
        sizes = [[B.dma_cache_decode_prefix_bytes(shape, n, 2048, p, 0) for p in (0, 1, 2, 5, 64)] for n in (1, 2, 7, 8, 9, 100, 256, 300)]
        for row in sizes:
            assert row == sorted(row)
        for column in zip(*sizes):
            assert list(column) == sorted(column)
