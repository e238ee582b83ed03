"""Calls of the same kernel from two threads at once, with different numbers of rows, each on a stream of its own."""
import os
import threading

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402
from decode_ref import freqs  # noqa: E402

pytestmark = pytest.mark.gpu


def test_weights_of_windows():
    gen = torch.Generator().manual_seed(7)
    table, pages, _ = R.paged(gen, [200], 16)
    table = table.cuda()
    kc = R.random_pool(seer, gen, pages, 2, 16, 128, 32)
    f = freqs(128).cuda()
    calls = []
    for S in (12, 40):
        q = torch.randn(1, 16, S, 128, generator=gen).to(torch.bfloat16).cuda()
        pos = (200 - S + torch.arange(S, dtype=torch.int32)).cuda()[None]
        lse = seer.paged_attn_q4(q, kc, kc, table, pos, inv_freq=f, want_lse=True)[1]
        w = torch.zeros(1, 2, 208).cuda()
        want = seer.kv_weights(q, kc, table, pos, lse, w.clone(), decay=0.0, inv_freq=f)
        calls.append((q, pos, lse, w, want))
    torch.cuda.synchronize()
    got, start = [[], []], threading.Barrier(2)

    def work(i):
        q, pos, lse, w, _ = calls[i]
        s = torch.cuda.Stream()
        start.wait()
        for _ in range(100):
            with torch.cuda.stream(s):
                out = w.clone()
            got[i].append(seer.kv_weights(q, kc, table, pos, lse, out, decay=0.0, inv_freq=f, stream=s))
        s.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for (_, _, _, _, want), out in zip(calls, got):
        assert len(out) == 100 and all(torch.equal(x, want) for x in out)
