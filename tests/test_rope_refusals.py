"""dma_rope and dma_cache_append_rope: what is refused, before any launch (so without a GPU)."""
import pytest

from paper_2508_02124_amd import binding as B

P = 0x1000  # an aligned address that a refused call never reads


def status(call):
    with pytest.raises(B.DmaError) as e:
        call()
    return e.value.status


def rope(**more):
    a = dict(T=8, n_docs=1, H_q=4, H_kv=2, d=64, Q=P, qs=256, K=P, ks=128, cu=P, pos=None, freqs=P, rot=64, Qo=2 * P, qos=256, Ko=3 * P, kos=128)
    a.update(more)
    shape = B.make_shape(a["T"], a["n_docs"], a["H_q"], a["H_kv"], a["d"], 1)
    return lambda: B.dma_rope(shape, a["Q"], a["qs"], a["K"], a["ks"], a["cu"], a["pos"], a["freqs"], a["rot"], False, False, a["Qo"], a["qos"],
                              a["Ko"], a["kos"], stream=0)


@pytest.mark.parametrize("more", [dict(T=0), dict(H_kv=3), dict(Q=None, K=None), dict(cu=None), dict(freqs=None), dict(rot=0), dict(rot=-16),
                                  dict(rot=80), dict(Q=P + 8), dict(Ko=P + 8), dict(Qo=None), dict(Ko=None), dict(qs=248), dict(kos=120), dict(qs=260),
                                  dict(qos=257), dict(Qo=P, qs=512), dict(Ko=P, kos=256)])
def test_rope_arguments(more):
    assert status(rope(**more)) == B.DMA_EINVAL


@pytest.mark.parametrize("more", [dict(rot=8), dict(rot=40), dict(d=96)])
def test_rope_sizes(more):
    assert status(rope(**more)) == B.DMA_EUNSUPPORTED


def append(n=4, reqs=4, **more):
    a = dict(Q=P, qs=256, K=P, ks=128, V=P, vs=128, W=P, A=P, z=None, slots=P, req=P, length=P, np=1, pl=P, of=P, freqs=P, rot=64, Qo=2 * P, pages=P)
    a.update(more)
    shape = B.make_cache_shape(reqs, 8, 8, 16, 4, 2, 64)
    return lambda: B.dma_cache_append_rope(shape, n, a["Q"], a["qs"], a["K"], a["ks"], a["V"], a["vs"], a["W"], a["A"], a["z"], a["slots"], a["req"],
                                           a["length"], a["np"], a["pl"], a["of"], a["freqs"], a["rot"], False, a["Qo"], a["pages"], stream=0)


@pytest.mark.parametrize("more", [dict(n=-1), dict(K=None), dict(V=None), dict(slots=None), dict(length=None), dict(pages=None), dict(A=None),
                                  dict(W=None), dict(Qo=None), dict(Q=P + 8), dict(Qo=P + 8), dict(K=P + 8), dict(V=P + 4), dict(pages=P + 8),
                                  dict(qs=248), dict(ks=100), dict(vs=127), dict(np=-1), dict(pl=None), dict(of=None), dict(n=5, req=None),
                                  dict(freqs=None), dict(rot=0), dict(rot=128), dict(Qo=P, qs=512)])
def test_append_arguments(more):
    assert status(append(**more)) == B.DMA_EINVAL


def test_append_sizes_and_no_rows():
    assert status(append(rot=24)) == B.DMA_EUNSUPPORTED
    append(n=0, Q=None, K=None, V=None, W=None, A=None, slots=None, length=None, Qo=None, pages=None)()
    with pytest.raises(OverflowError):
        append(rot=1 << 32)()
