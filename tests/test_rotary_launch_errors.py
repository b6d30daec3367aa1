"""Every launch of the rotary calls and of the decode behind prefixes is reported if it fails (the stand-in of test_launch_errors, in a process of its
own)."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2508_02124_amd import binding as B
from test_launch_errors import ROOT, STAND_IN

# Shapes that take each route: one launch of rows and several (more than 2^22), pairs of either kind; lists in one launch, in slices, in
# several launches of slices, of prefixes only and of rows too; many and few pairs, windows that keep everything, no prefixes.
CALLS = r"""
import ctypes, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_2508_02124_amd import binding as B
P = 0x1000  # (never dereferenced: nothing runs)
launches = set()

def each_fails(name, call):
    runtime.start(0)
    call()
    n = runtime.launched()
    assert n > 0
    launches.add((name, n))
    for i in range(1, n + 1):
        runtime.start(i)
        try:
            call()
            print(f"LOST: {name}, launch {i} of {n}")
        except B.DmaError as e:
            assert e.status == B.DMA_EHIP, (name, i, e)

for T, d, next in ((1, 64, False), (5000, 128, True), (3 << 22, 256, False)):
    for dtype in (0, 1):
        s = B.make_shape(T, 1, 8, 2, d, 1, dtype=dtype)
        each_fails("rope", lambda: B.dma_rope(s, P, 8 * d, P, 2 * d, P, None, P, 32, next, False, 2 * P, 8 * d, 3 * P, 2 * d, stream=0))
        c = B.make_cache_shape(4, 100, 10, 64, 8, 2, d, dtype=dtype)
        each_fails("append", lambda: B.dma_cache_append_rope(c, T, P, 8 * d, P, 2 * d, P, 2 * d, P, P, None, P, P, P, 2, P, P, P, 32, next, 2 * P, P,
                                                             stream=0))
for ps, k, max_pages, H_q, d, n_rows, n_prefixes, max_len, max_prefix in (
        (16, 64, 100, 8, 64, 4, 2, 0, 0), (32, 64, 100, 8, 128, 4, 0, 0, 0), (64, 300, 100, 8, 256, 200, 3, 1000, 0), (64, 9000, 100, 8, 64, 4, 1, 0, 0),
        (64, 2048, 1000, 8, 128, 4, 2, 0, 0), (32, 2048, 1000, 8, 64, 4, 2, 2000, 0), (16, 512, 4000, 32, 64, 300, 600, 0, 0),
        (64, 512, 1000, 32, 64, 300, 2, 0, 4000), (64, 512, 190, 32, 64, 600, 300, 0, 0)):
    for dtype in (0, 1):
        s = B.make_cache_shape(4000, 5000, max_pages, ps, H_q, 2, d, dtype=dtype, max_len=max_len)
        each_fails(f"decode {n_rows} {n_prefixes}", lambda: B.dma_cache_decode_prefix(s, n_rows, k, 0.0, P, H_q * d, P, P, P, P, n_prefixes, max_prefix, P, P,
                                                                                     P, P, P, P, 1 << 50, stream=0))
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
    assert "LOST" not in r.stdout, r.stdout
    for some in ("('rope', 1)", "('rope', 3)", "('append', 3)", "('decode 4 2', 4)", "('decode 4 2', 5)", "('decode 4 0', 3)", "('decode 300 600', 9)",
                 "('decode 600 300', 4)"):
        assert some in r.stdout, (some, r.stdout)
