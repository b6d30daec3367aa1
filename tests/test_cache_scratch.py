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
for max_pages, k in ((10, 100), (10, 5000)):
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
