"""Windows of tokens whose rows take more than 64 KB of LDS (kv_weights), and their attention, captured and replayed."""
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402
from decode_ref import freqs  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,dtype", [("q4", torch.bfloat16), ("q4", torch.float32), ("bf16", torch.bfloat16)])
def test_a_captured_window(kind, dtype):
    gen = torch.Generator().manual_seed(1)
    S, page, n = 40, 16, 500
    table, pages, _ = R.paged(gen, [n, n], page)
    table, f = table.cuda(), freqs(128).cuda()
    if kind == "q4":
        kc, attn = R.random_pool(seer, gen, pages, 2, page, 128, 32), seer.paged_attn_q4
    else:
        kc, attn = torch.randn(pages, 2, page, 128, generator=gen).to(dtype).cuda(), seer.paged_attn

    def step(q, pos, w):
        o, lse = attn(q, kc, kc, table, pos, inv_freq=f, want_lse=True)
        return o, lse, seer.kv_weights(q, kc, table, pos, lse, w, decay=0.5, inv_freq=f)

    def draw(i):
        g = torch.Generator().manual_seed(i)
        last = torch.randint(S, n, (2, 1), generator=g)
        return (torch.randn(2, 16, S, 128, generator=g).to(dtype).cuda(), (last - S + torch.arange(S)).to(torch.int32).cuda(),
                torch.rand(2, 2, table.shape[1] * page, generator=g).cuda())

    args = draw(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*draw(9))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*args)
    for i in range(4):
        for a, x in zip(args, draw(i)):
            a.copy_(x)
        graph.replay()
        want = step(*draw(i))
        torch.cuda.synchronize()
        for a, x in zip(out, want):
            assert torch.equal(a, x)
