"""Every launch of the paged cache's calls is reported if it fails (the stand-in of test_launch_errors, in a process of its own)."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2508_02124_amd import binding as B
from test_launch_errors import ROOT, STAND_IN

# Shapes that take each route: many and few rows of a step, short rows, rows in slices, windows that keep everything, one part of a
# list and several.
CALLS = r"""
import ctypes, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_2508_02124_amd import binding as B
P = 0x1000  # (never dereferenced: nothing runs)
launches = set()
for n_reqs, max_pages, ps, k, n_rows, d, dtype in ((4, 100, 16, 64, 4, 64, 0), (4, 100, 64, 300, 4, 128, 0), (4, 1000, 64, 2048, 4, 128, 1),
                                                   (4, 1000, 16, 2048, 4, 256, 0), (4, 10, 64, 5000, 4, 128, 0), (2000, 10, 64, 100, 5000, 64, 1)):
    s = B.make_cache_shape(n_reqs, 5000, max_pages, ps, 8, 2, d, dtype=dtype)
    calls = {
        "reset": lambda: B.dma_cache_reset(s, P, P, P, stream=0),
        "assign": lambda: B.dma_cache_assign(s, n_rows, *[P] * 9, stream=0),
        "append": lambda: B.dma_cache_append(s, n_rows, P, 2 * d, P, 2 * d, P, P, None, P, P, stream=0),
        "read": lambda: B.dma_cache_read(s, n_rows, *[P] * 5, stream=0),
        "decode": lambda: B.dma_cache_decode(s, n_rows, k, 0.0, P, 8 * d, *[P] * 8, 1 << 40, stream=0),
    }
    for name, call in calls.items():
        runtime.start(0)
        call()
        n = runtime.launched()
        assert n > 0
        launches.add((name, n))
        for i in range(1, n + 1):
            runtime.start(i)
            try:
                call()
                print(f"LOST: {name} n_rows={n_rows} k={k} ps={ps}, launch {i} of {n}")
            except B.DmaError as e:
                assert e.status == B.DMA_EHIP, (name, i, e)
print("calls", sorted(launches))
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_failed_launch_is_reported(tmp_path):
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    source, stand_in, calls = tmp_path / "stand_in.cpp", tmp_path / "stand_in.so", tmp_path / "calls.py"
    source.write_text(STAND_IN)
    calls.write_text(CALLS)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(source), "-o", str(stand_in)], check=True)
    r = subprocess.run([sys.executable, str(calls), str(stand_in), ROOT], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "LOST" not in r.stdout and "('decode', 4)" in r.stdout and "('assign', 2)" in r.stdout, r.stdout
