"""The selecting launches of dma_cache_decode_prefix make the lists of every (row, head) and (prefix, head) pair once, however many launches
share the scratch (over a stand-in for the runtime's launch functions, which runs nothing and writes down what each launch is given; in a
process of its own)."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2508_02124_amd import binding as B
from test_launch_errors import ROOT

# The kernels' names come with their registration, their arguments with each launch.
STAND_IN = r"""
#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
struct dim3 { unsigned x, y, z; };
struct Rows { const int32_t *table, *row_req, *row_len; int n_rows, k, kcap; };
struct Work { void *counts, *listed, *bounds; int room, parts, first, pairs; };
struct Set { Rows rows; Work sw; int32_t* list; uint32_t* keys; int wgs; };
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
static dim3 g_grid;
extern "C" {
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[host] = name; }
int __hipPushCallConfiguration(dim3 grid, dim3, size_t, void*) { g_grid = grid; return 0; }
int __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, void** stream) {
  *grid = g_grid;
  *block = {1, 1, 1};
  *lds = 0;
  *stream = nullptr;
  return 0;
}
int hipLaunchKernel(const void* host, dim3 grid, dim3, void** args, size_t, void*) {
  const char *name = names()[host].c_str(), *at = strstr(name, "prefix_select_kernelILi");
  const bool slice = !at && (at = strstr(name, "prefix_slice_kernelILi"));
  if (!at) return 0;
  // <S, SLICED, GROUP>, or <S>: the digits behind "Li" and "Lb"
  const char* b = strstr(at, "ELb");
  const int sliced = slice ? 1 : b[3] - '0', group = slice ? 0 : b[7] - '0';
  printf("%s %d %d grid %u", slice ? "slice" : "select", sliced, group, grid.x);
  for (int i = slice ? 1 : 2; i < (slice ? 3 : 4); i++) {
    const Set& x = *(const Set*)args[i];
    printf(" | %d %d %d %d", x.wgs, x.sw.parts, x.sw.first, x.sw.pairs);
  }
  printf("\n");
  return 0;
}
int hipGetLastError() { return 0; }
}
"""

CALLS = r"""
import ctypes, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_2508_02124_amd import binding as B
P = 0x1000  # (never dereferenced: nothing runs)
H_q, ps, k, max_tokens, n_rows, n_prefixes, max_len, max_prefix = (int(x) for x in sys.argv[3:])
s = B.make_cache_shape(4096, 4096, max_tokens // ps, ps, H_q, 1, 64, max_len=max_len)
B.dma_cache_decode_prefix(s, n_rows, k, 0.0, P, H_q * 64, P, P, P, P, n_prefixes, max_prefix, P, P, P, P, P, P, 1 << 50, stream=0)
"""

# heads, page size, window, longest request, rows, prefixes, bounds on own keys and prefixes (0: none)
CASES = {
    "few": (32, 64, 512, 8192, 20, 3, 0, 0),
    "rows, short": (32, 64, 512, 8192, 512, 1, 0, 0),
    "rows, short, a prompt": (32, 32, 512, 12288, 4000, 1, 4000, 0),
    "prefixes, short": (32, 16, 300, 4096, 40, 300, 0, 0),
    "both, short": (32, 64, 512, 8192, 300, 400, 0, 0),
    "rows, long": (32, 64, 512, 65536, 300, 1, 0, 4000),
    "prefixes, long": (32, 64, 512, 65536, 40, 300, 2500, 0),
    "both, long": (32, 16, 512, 65536, 300, 700, 0, 0),
    "rows all kept, prefixes long": (16, 64, 4096, 65536, 1000, 600, 4000, 0),
    "everything kept": (32, 64, 8192, 8192, 300, 300, 0, 0),
}


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    d = tmp_path_factory.mktemp("prefix_launches")
    (d / "stand_in.cpp").write_text(STAND_IN)
    (d / "calls.py").write_text(CALLS)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", str(d / "stand_in.cpp"), "-o", str(d / "stand_in.so")], check=True)
    return d


@pytest.mark.parametrize("name", CASES)
def test_every_pair_has_its_list_once(stand_in, name):
    H_q, ps, k, longest, n_rows, n_prefixes, max_len, max_prefix = CASES[name]
    r = subprocess.run([sys.executable, str(stand_in / "calls.py"), str(stand_in / "stand_in.so"), ROOT, *map(str, CASES[name])], capture_output=True,
                       text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr
    launches = [line.split() for line in r.stdout.splitlines() if line.split()[:1] in (["select"], ["slice"])]
    assert launches and launches[0][:3:2] == ["select", "1"] and all(x[2] == "0" for x in launches[1:])   # (the first one orders the rows)
    listed = (max_len or longest) > max(k, 2048)            # rows of more than k keys of their own have lists
    want = (n_prefixes * H_q, n_rows * H_q if listed else 0)
    for of_set in range(2):
        made, ranked, long = [], [], False
        for x in launches:
            wgs, parts, first, pairs = (int(y) for y in x[6 + 5 * of_set:10 + 5 * of_set])
            if wgs == 0:
                continue
            assert first >= 0 and wgs == pairs * max(1, parts)
            if x[0] == "slice":
                ranked.append((first, pairs))
                continue
            long |= parts > 0
            assert x[1] == "1" or first == 0                # without slices there is no share of the scratch: all pairs are in one launch
            made.append((first, pairs))
        at = 0
        for first, pairs in made:
            assert first == at
            at += pairs
        assert at == want[of_set]
        assert ranked == (made if long else [])
    for x in launches:
        assert int(x[4]) == int(x[2]) + int(x[6]) + int(x[11])
