"""Sequences without keys over a cache in 4 bits, whose table rows are narrower than a tile of keys."""
import math
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402
from decode_ref import assert_rounded  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,wide", [(1, 3), (2, 1), (5, 2), (16, 1), (16, 6), (24, 2), (64, 1)])
def test_the_last_sequence_is_empty(dtype, page, wide):
    """The table stands in a wider tensor, whose entries to its right and behind it name a page of NaN: what lies beyond
    a row's entries does not reach any output."""
    gen = torch.Generator().manual_seed(page + wide)
    room = page * wide
    lengths = [room, 0, max(room - 1, 1), 0]
    tight, pages, spare = R.paged(gen, lengths, page, wide=wide)
    kc, vc = (R.random_pool(seer, gen, pages, 2, page, 64, 32) for _ in range(2))
    for pool in (kc, vc):
        pool.params[spare] = math.nan
    whole = torch.full((600, wide + 600), spare[0], dtype=torch.int32)
    whole[:4, :wide] = tight
    table = whole.cuda()[:4, :wide]
    q = torch.randn(4, 4, 2, 64, generator=gen).to(dtype)
    pos = torch.tensor([[n - 2, n - 1] if n else [-1, -9] for n in lengths], dtype=torch.int32)
    o, lse = seer.paged_attn_q4(q.cuda(), kc, vc, table, pos.cuda(), want_lse=True)
    ro, rl, eo, el = R.attend(q, kc, vc, tight, page, pos, 0.0)
    none = (pos < 0)[:, None].expand(4, 4, 2)
    assert torch.equal(lse.cpu() == -math.inf, none) and not bool(o.cpu()[none].any())
    assert bool(((lse.cpu().double() - rl).abs()[~none] <= (el + R.U * rl.abs())[~none]).all())
    assert_rounded(o, ro, eo, "o")
