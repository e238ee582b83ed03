"""Paged attention over a table with room for 2^30 keys a row: a unit of the work is then more than a
tile for each wavefront, so that the weights of all units stay below 2^30, whatever the lengths are."""
import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")

from decode_ref import freqs, make_cache  # noqa: E402
from test_gpu_paged_attn import TYPES, check  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("Hkv,tokens", [(4, 1), (2, 2), (1, 1)])
def test_units_of_several_tiles(dtype, Hkv, tokens):
    """64 sequences on the same pages, of lengths around the edges of units of 128, 256 and 512 keys: with 4, 2 and 1 KV
    heads 2^23 units of 128 keys a row are 2^31, 2^30 and 2^29, so units are of 512, 256 and 128 (fp32, from 64: the same)."""
    print(f"[paged] wide table {dtype} {Hkv} {tokens}", flush=True)
    gen = torch.Generator().manual_seed(Hkv)
    lengths = [3000, 0, 1, 2, 31, 33, 127, 128, 129, 255, 256, 257, 511, 512, 513, 639, 640, 641, 767, 768, 769, 1023, 1024, 1025,
               1535, 1536, 1537, 2047, 2048, 2049, 2559, 2561]
    lengths += [int(x) for x in torch.randint(1, 1400, (64 - len(lengths),), generator=gen)]
    kc, vc, table = make_cache(gen, [max(lengths)], 64, Hkv, 64, TYPES[dtype], wide=1 << 24, fill=float("nan"))
    q = torch.randn(64, 2 * Hkv, tokens, 64, generator=gen).to(TYPES[dtype])
    pos = (torch.tensor(lengths)[:, None] - tokens + torch.arange(tokens)).to(torch.int32)
    wide = table.cuda().expand(64, -1)
    assert wide.stride(0) == 0
    o, lse = check(q, kc, vc, _Shared(table, wide), pos)
    check(q, kc, vc, _Shared(table, wide), pos, rope=(freqs(64), 1.0, False))
    # a table that is as wide as the longest sequence needs gives the same up to the order of the sums
    narrow = table[:, :48].expand(64, -1).contiguous()
    o2, lse2 = check(q, kc, vc, narrow, pos)
    assert torch.equal(lse.isinf(), lse2.isinf())


class _Shared:
    """One row of a table for every sequence: as `check` indexes it and moves it to the GPU."""

    def __init__(self, row, wide):
        self.row, self.wide, self.shape = row, wide, wide.shape

    def __getitem__(self, b):
        return self.row[0]

    def cuda(self):
        return self.wide
