"""The scratch of a decode over the paged cache, without a GPU: its size, and the launches that share it (over the stand-in of
test_launch_errors, which runs nothing, in a process of its own)."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2508_02124_amd import binding as B
from test_launch_errors import ROOT, STAND_IN

HEAD = r"""
import ctypes, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_2508_02124_amd import binding as B
P = 0x1000  # (never dereferenced: nothing runs)
"""


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return B.lib()


def over_stand_in(tmp_path, calls):
    source, stand_in, script = tmp_path / "stand_in.cpp", tmp_path / "stand_in.so", tmp_path / "calls.py"
    source.write_text(STAND_IN)
    script.write_text(HEAD + calls)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(source), "-o", str(stand_in)], check=True)
    r = subprocess.run([sys.executable, str(script), str(stand_in), ROOT], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


needs_compiler = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")


@needs_compiler
def test_no_scratch_needs_no_address(tmp_path):
    """An allocation of no bytes has no address."""
    out = over_stand_in(tmp_path, r"""
for max_pages, k in ((10, 100), (4, 5000)):
    s = B.make_cache_shape(400, 4000, max_pages, 64, 8, 2, 128)
    assert B.dma_cache_decode_bytes(s, 400, k) == 0
    runtime.start(0)
    B.dma_cache_decode(s, 400, k, 0.0, P, 1024, *[P] * 7, None, 0, stream=0)
    print("launches", runtime.launched())
s = B.make_cache_shape(4, 4000, 1000, 64, 8, 2, 128)
need = B.dma_cache_decode_bytes(s, 4, 2048)
assert need > 0
for ws, size in ((None, need), (P, need - 1), (None, 0)):
    runtime.start(0)
    try:
        B.dma_cache_decode(s, 4, 2048, 0.0, P, 1024, *[P] * 7, ws, size, stream=0)
        print("TAKEN", ws, size)
    except B.DmaError as e:
        assert e.status == B.DMA_EWORKSPACE and runtime.launched() == 0
""")
    assert "TAKEN" not in out and out.split() == ["launches", "2", "launches", "1"], out


def test_size_of_the_scratch():
    """Lists of 8192 keys of 8 bytes for each (row, head), but 256 MiB at most, with 512 bytes of counts and 16 of bounds for 8192 pairs at
    most; before them the partial outputs of fewer than 512 lists.  None of the lists where no row can have more than 12288 keys."""
    s = B.make_cache_shape(4096, 100000, 16384, 64, 32, 8, 128)
    for n_rows in (8, 128, 129, 256, 257, 1024, 4096):
        pairs = 32 * n_rows
        lists = min(65536 * pairs, 256 << 20) + (512 + 16) * min(pairs, 8192)
        assert lists <= B.dma_cache_decode_bytes(s, n_rows, 2048) <= lists + 512 * 130 * 4 + 1024, n_rows
    for n_rows in (1, 3, 7, 8, 9, 100, 127, 128, 129, 255, 256, 257, 300, 511, 513, 2047, 5000, 16375):
        for d, k in ((64, 1), (256, 2048), (128, 100000)):
            for max_len in (0, 12288, 12289, 100000):
                t = B.make_cache_shape(4096, 100000, 16384, 64, 32, 8, d, max_len=max_len)
                size = B.dma_cache_decode_bytes(t, n_rows, k)
                assert size < (1 << 20 if max_len == 12288 else 261 << 20), (n_rows, d, k, max_len)


@needs_compiler
def test_launches_that_share_the_scratch(tmp_path):
    """More pairs than there is room for: a selection in several launches, each failed one reported."""
    out = over_stand_in(tmp_path, r"""
s = B.make_cache_shape(4096, 100000, 16384, 64, 32, 8, 128)
for n_rows, want in ((256, 2 + 1), (257, 2 * 2 + 1), (513, 3 * 2 + 1), (3000, 12 * 2 + 1)):
    size = B.dma_cache_decode_bytes(s, n_rows, 2048)
    call = lambda: B.dma_cache_decode(s, n_rows, 2048, 0.0, P, 4096, *[P] * 8, size, stream=0)
    runtime.start(0)
    call()
    assert runtime.launched() == want, (n_rows, runtime.launched())
    for i in range(1, want + 1):
        runtime.start(i)
        try:
            call()
            print(f"LOST: launch {i} of {want}")
        except B.DmaError as e:
            assert e.status == B.DMA_EHIP
""")
    assert "LOST" not in out, out


def test_more_rows_need_no_less():
    """A program may keep the scratch of its largest step for all of them."""
    for H_q, H_kv, d in ((32, 8, 128), (1, 1, 64), (8, 2, 256), (300, 3, 64)):
        for max_pages, k in ((16384, 2048), (10, 300), (10, 5000), (100, 4000), (16384, 100000), (40, 257)):
            s, last = B.make_cache_shape(4096, 100000, max_pages, 64, H_q, H_kv, d), 0
            for n_rows in [*range(1, 400), *range(400, 3000, 37)]:
                size = B.dma_cache_decode_bytes(s, n_rows, k)
                if size == 0 and (n_rows + 8) * H_q * -(-min(k, max_pages * 64) // 256) >= 1 << 22:
                    break                            # (more rows than a call takes)
                assert size >= last, (H_q, max_pages, k, n_rows, last, size)
                last = size
