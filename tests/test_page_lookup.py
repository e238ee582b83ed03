"""Where the kernels look up a key's page, by the functions that they use, compiled for the host (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

seer = pytest.importorskip("paper_2410_13276_amd")
from paper_2410_13276_amd import build  # noqa: E402

HIPCC = shutil.which(build.HIPCC)
if HIPCC is None:
    pytest.skip("no hipcc", allow_module_level=True)

SOURCE = """
#include <cstdio>
#include "paged_common.h"
int main() {
  int page, n;
  while (std::scanf("%d %d", &page, &n) == 2) {
    const seer::FastDiv f = seer::fast_div(page);
    std::printf("%d %d\\n", n >= 0 ? seer::fast_quot(f, n) : 0, seer::last_page_of(f, n));
  }
}
"""
PAGES = [1, 2, 3, 5, 7, 12, 16, 24, 64, 100, 256, 1000, 65536, (1 << 30) - 1, 1 << 30]


@pytest.fixture(scope="module")
def looked_up(tmp_path_factory):
    d = tmp_path_factory.mktemp("lookup")
    src = d / "lookup.hip"
    src.write_text(SOURCE)
    subprocess.run([HIPCC, *build.FLAGS, "--offload-host-only", str(src), "-o", str(d / "lookup")], check=True, capture_output=True)

    def ask(pairs):
        out = subprocess.run([str(d / "lookup")], input="".join(f"{p} {n}\n" for p, n in pairs), text=True, check=True,
                             capture_output=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return ask


def test_quotients(looked_up):
    pairs = [(p, n) for p in PAGES for x in (0, 1, p - 1, p, p + 1, 2 * p, 12345, 123456789, (1 << 30) - 1, (1 << 30), (1 << 31) - 1)
             for n in (x,) if 0 <= n < 1 << 31]
    for (p, n), (q, _) in zip(pairs, looked_up(pairs)):
        assert q == n // p, (p, n)


def test_look_ups_stay_in_the_row(looked_up):
    """The last page of a run of keys is the one of its last key, and the first entry of the row where the run has none (a
    sequence whose positions are all negative): look-ups of the tiles behind the run are held to it."""
    pairs = [(p, n) for p in PAGES for n in (0, 1, 2, p - 1, p, p + 1, 511, 512, 513, 1 << 30) if n <= 1 << 30]
    for (p, n), (_, last) in zip(pairs, looked_up(pairs)):
        assert last == max(n - 1, 0) // p, (p, n)
        wide = max(-(-n // p), 1)  # the narrowest table that holds the sequence
        for key in (0, 63, 511, n + 511):
            assert 0 <= min(key // p, last) < wide
