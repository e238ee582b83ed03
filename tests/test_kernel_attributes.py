"""What a call sets on a kernel, which is the process's and not the call's: two threads may be in calls of the same kernel at once, with
different numbers of rows.  The runtime's functions that the library calls are stood in for by ones that note their arguments (no GPU
needed, nothing is launched)."""
import os
import shutil
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)
CC = shutil.which("gcc")
if CC is None:
    pytest.skip("no gcc", allow_module_level=True)

HERE = os.path.dirname(os.path.abspath(__file__))

STANDIN = r"""
#include <stddef.h>
#include <stdio.h>
typedef struct { unsigned x, y, z; } d3;
static d3 grid, block;
static size_t shared;
static void* at;
int hipFuncSetAttribute(const void* f, int attr, int value) { printf("set %p %d\n", f, value); return 0; }
int __hipPushCallConfiguration(d3 g, d3 b, size_t s, void* st) { grid = g, block = b, shared = s, at = st; return 0; }
int __hipPopCallConfiguration(d3* g, d3* b, size_t* s, void** st) { *g = grid, *b = block, *s = shared, *st = at; return 0; }
int hipLaunchKernel(const void* f, d3 g, d3 b, void** args, size_t s, void* st) { printf("run %p %zu\n", f, s); return 0; }
int hipGetLastError(void) { return 0; }
int hipPeekAtLastError(void) { return 0; }
"""

# calls of few rows and of many, whose rows take the LDS from some KB to all that the kernel uses
CALLS = r"""
import ctypes as C, os, sys
sys.path[:0] = [sys.argv[2], os.path.dirname(sys.argv[2])]
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
import paper_2410_13276_amd as seer
from paper_2410_13276_amd import cache
import test_cache_abi as A
L = C.CDLL(seer.LIB_PATH)
fn = L.seer_kv_weights
fn.argtypes, fn.restype = cache.SIGS["seer_kv_weights"]
for D in (64, 128):
    for group, dtypes in ((0, (0, 1)), (32, (0, 1)), (64, (0, 1))):
        for dtype in dtypes:
            for turns in (False, True):
                for tokens in (1, 4, 8, 12, 16, 24, 40, 64, 200, 24, 1):
                    c = A.make_cache(H=2, D=D, dtype=dtype, group=group, rows=4, wide=64)
                    w = cache._WEIGHTS.pack(A.FAKE, A.FAKE, 2048, 1024, 2048, 1024, 1024, 1.0)
                    q = A.queries(B=2, Hq=8, S=tokens, dtype=dtype, H=2, D=D, ps=tokens)
                    s = fn(c, q, A.rope(rot=D) if turns else None, 0.0, A.FAKE, A.FAKE, None, A.FAKE, w, None)
                    assert s == 0, (s, D, group, dtype, turns, tokens)
"""


def test_the_largest_lds_is_set_alike_by_all_calls(tmp_path):
    src, lib, calls = (tmp_path / n for n in ("standin.c", "standin.so", "calls.py"))
    src.write_text(STANDIN)
    calls.write_text(CALLS)
    subprocess.run([CC, "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    r = subprocess.run([sys.executable, str(calls), str(lib), HERE], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    value, runs = {}, 0
    for line in r.stdout.splitlines():
        what, kernel, n = line.split()
        if what == "set":
            assert value.setdefault(kernel, int(n)) == int(n), (kernel, value[kernel], n)
        elif what == "run":
            runs += 1
            # (64 KB need no setting, the kernel's own static arrays among them)
            assert int(n) <= value.get(kernel, 64 << 10), (kernel, n)
    assert runs == 2 * 3 * 2 * 2 * 11 and len(value) > 4
