"""The largest calls that the cache's checks let through: their launches keep within what the runtime takes (less than 2^32 threads a
dimension, 65535 workgroups in y).  The runtime's functions are stood in for, nothing is launched (no GPU needed)."""
import subprocess
import sys

import pytest

from test_kernel_attributes import CC, HERE, STANDIN

CALLS = r"""
import ctypes as C, os, sys
sys.path[:0] = [sys.argv[2], os.path.dirname(sys.argv[2])]
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
import paper_2410_13276_amd as seer
from paper_2410_13276_amd import cache
import test_cache_abi as A
L = C.CDLL(seer.LIB_PATH)
def call(name, *args):
    fn = getattr(L, name)
    fn.argtypes, fn.restype = cache.SIGS[name]
    print("call", name, fn(*args), flush=True)
F = A.FAKE
TOP = 1 << 40
for H, T in ((1, 1 << 27), (65535, 1 << 27), (65535, 1), (65535, 2000)):
    for D in (64, 128):
        for group, dtype in ((32, 0), (64, 1), (0, 0), (0, 1)):
            c = A.make_cache(H=H, D=D, dtype=dtype, group=group, rows=4, wide=64, st=(TOP, 1 << 30, 1 << 10), pst=(TOP, 1 << 30, 1 << 10))
            t = A.tokens(B=1, S=T, dtype=dtype, H=H, D=D, ks=(0, TOP, 128))
            call("seer_kv_read", c, t, F, F, F, None, None)
            if group:
                call("seer_kv_append_q4", c, t, None, F, F, F, None, None, None)
for H, B, S, Hq in ((1, 1, 1 << 23, 1), (1, 1 << 23, 1, 1), (65535, 128, 1, 65535), (1, 1, 1 << 19, 16), (65535, 1, 1, 65535)):
    for group, dtype in ((32, 0), (64, 1), (0, 0), (0, 1)):
        c = A.make_cache(H=H, dtype=dtype, group=group, rows=B, page=1 << 10, wide=1 << 20, ts=0, st=(1 << 35, 1 << 30, 1 << 10), pst=(1 << 32, 1 << 30, 1 << 10))
        q = A.queries(B=B, Hq=Hq, S=S, dtype=dtype, H=H, qs=(0, 0, 0), os_=(TOP, 1 << 35, 128), ps=0)
        w = cache._WEIGHTS.pack(F, F, 1 << 50, 1 << 31, 1 << 50, 1 << 31, (1 << 31) - 1, 1.0)
        call("seer_kv_weights", c, q, None, 0.0, F, F, None, F, w, None)
        if group:
            call("seer_paged_attn_q4", c, q, None, 0.0, F, F, None, F, F, F, 1 << 62, None)
for H, B in ((1, 1 << 22), (1, (1 << 22) - 1), (64, 1 << 16), (65535, 63), (65535, 1), (1, 1)):
    for wide in (1, 1 << 20):
        for keep in (1, 1024):
            c = A.make_cache(H=H, group=0, rows=B, page=1 << 10, wide=wide, ts=0, st=(TOP, 1 << 30, 1 << 10))
            e = cache._EVICTION.pack(B, keep, 0, 0, F, F, F, 0, 1, 1 << 20, 1 << 20, 0, F, F + 4096, 1 << 50, 1 << 30, 1 << 50, 1 << 30, F)
            call("seer_kv_evict", c, e, F, 1 << 62, None)
"""


def test_launches_at_the_limits(tmp_path):
    src, lib, calls = (tmp_path / n for n in ("standin.c", "standin.so", "calls.py"))
    src.write_text(STANDIN.replace(r'printf("run %p %zu\n", f, s)',
                                   r'printf("run %u %u %u %u %u %u\n", g.x, g.y, g.z, b.x, b.y, b.z), fflush(stdout)'))
    calls.write_text(CALLS)
    subprocess.run([CC, "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    r = subprocess.run([sys.executable, str(calls), str(lib), HERE], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    runs, done = [], {}
    for line in r.stdout.splitlines():
        what, *x = line.split()
        if what == "run":
            runs.append([int(y) for y in x])
        elif what == "call":
            name, status = x[0], int(x[1])
            assert status in (0, 2), (name, status)  # served, or refused as unsupported
            assert bool(runs) == (status == 0), (name, status, runs)
            for g in runs:
                assert all(0 < a * b < 1 << 32 for a, b in zip(g[:3], g[3:])) and g[1] <= 65535 and g[2] <= 65535, (name, g)
            done[name] = done.get(name, 0) + (status == 0)
            runs = []
    assert len(done) == 5 and min(done.values()) >= 8, done
