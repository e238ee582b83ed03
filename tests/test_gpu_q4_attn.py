"""Attention over a cache in 4 bits against the 64-bit form over the values that the cache stands for."""
import math
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402
from decode_ref import assert_rounded, freqs  # noqa: E402

pytestmark = pytest.mark.gpu


def check(gen, dtype, Hq, Hkv, D, group, page, lengths, S=1, order="phsd", turn=None, scale=0.0, wide=None, pos=None,
          rope_pos=None, mend=None):
    """One call on sequences whose last token is the last of `lengths`; returns (o, lse)."""
    B = len(lengths)
    table, pages, _ = R.paged(gen, lengths, page, wide=wide)
    kc, vc = (R.random_pool(seer, gen, pages, Hkv, page, D, group, order) for _ in range(2))
    q = (1.5 * torch.randn(B, Hq, S, D, generator=gen)).to(dtype)
    if pos is None:
        pos = (torch.tensor(lengths)[:, None] - S + torch.arange(S)).to(torch.int32)
    if mend is not None:
        mend(q, kc, vc, table)
    how = {}
    if turn is not None:
        how = dict(inv_freq=turn[0].cuda(), rope_scale=turn[1], interleaved=turn[2])
        if rope_pos is not None:
            how["rope_positions"] = rope_pos.cuda()
    o, lse = seer.paged_attn_q4(q.cuda(), kc, vc, table.cuda(), pos.cuda(), sm_scale=scale, want_lse=True, **how)
    ro, rl, eo, el = R.attend(q, kc, vc, table, page, pos, scale, turn, rope_pos)
    none = rl == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, none)
    assert bool((o.cpu()[none] == 0).all())
    d = (lse.cpu().double() - rl).abs()
    assert bool((d[~none] <= el[~none] + R.U * rl[~none].abs()).all()), float((d - el)[~none].max())
    assert_rounded(o, ro, eo, "o")
    return o, lse


SHAPES = [(2, 1, 64, 32), (2, 1, 64, 64), (4, 4, 64, 32), (8, 2, 128, 32), (8, 2, 128, 64), (7, 1, 128, 32), (12, 1, 128, 32),
          (24, 1, 128, 64), (20, 1, 64, 64)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,D,group", SHAPES)
def test_one_token(dtype, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(Hq + D + group)
    check(gen, dtype, Hq, Hkv, D, group, 16, [1, 63, 64, 65, 300], wide=20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,D,group", SHAPES)
def test_drafted_tokens_rotated(dtype, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(Hq + D + group + 1)
    check(gen, dtype, Hq, Hkv, D, group, 24, [130, 3, 66], S=3, order="pshd", turn=(freqs(D, 500000.0), 1.1, False))


@pytest.mark.parametrize("page", [1, 5, 8, 16, 48, 64, 100, 256])
@pytest.mark.parametrize("order", ["phsd", "pshd"])
def test_page_sizes(page, order):
    gen = torch.Generator().manual_seed(page)
    check(gen, torch.bfloat16, 8, 2, 128, 32, page, [200, 7, 131], order=order)


@pytest.mark.parametrize("S,Hq,Hkv,D,group", [(2, 4, 2, 128, 32), (8, 2, 1, 128, 32), (17, 2, 1, 64, 32), (5, 7, 1, 128, 64)])
def test_numbers_of_tokens(S, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(S)
    check(gen, torch.bfloat16, Hq, Hkv, D, group, 16, [S, S + 70, 300], S=S)


@pytest.mark.parametrize("rot,interleaved", [(16, False), (96, False), (128, True), (32, True)])
def test_rotation_at_other_positions(rot, interleaved):
    """Slots are no positions once keys were evicted."""
    gen = torch.Generator().manual_seed(rot)
    at = torch.randint(0, 200000, (2, 2), generator=gen).to(torch.int32)
    check(gen, torch.bfloat16, 8, 2, 128, 32, 16, [90, 40], S=2, turn=(freqs(rot, 10000.0), 1.0, interleaved), rope_pos=at)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_without_keys(dtype):
    """Negative positions, tables without pages, holes between pages: and NaN in every slot that is not seen."""
    gen = torch.Generator().manual_seed(2)
    lengths = [0, 40, 33, 50, 20]
    pos = torch.tensor([[-1, -1], [-1, 39], [31, 32], [10, -7], [18, 19]], dtype=torch.int32)

    def mend(q, kc, vc, table):
        table[2] = -1
        table[3, 0] = 10 ** 6
        real = torch.zeros(kc.codes.shape[0], kc.codes.shape[2], dtype=torch.bool)
        for b in range(5):
            n = int(pos[b].max()) + 1
            for t in range(max(n, 0)):
                p = int(table[b, t // 16])
                if 0 <= p < real.shape[0]:
                    real[p, t % 16] = True
        for pool in (kc, vc):
            pool.params.copy_(torch.where(real[:, None, :, None, None].cuda(), pool.params, math.nan))

    check(gen, dtype, 4, 2, 64, 32, 16, lengths, S=2, wide=6, pos=pos, mend=mend)


def test_unseen_drafts_hold_anything():
    """What a later drafted token holds does not reach the ones before it, be it NaN."""
    gen = torch.Generator().manual_seed(4)
    table, pages, _ = R.paged(gen, [70], 16)
    kc, vc = (R.random_pool(seer, gen, pages, 1, 16, 128, 32) for _ in range(2))
    q = torch.randn(1, 4, 3, 128, generator=gen).to(torch.bfloat16).cuda()
    pos = torch.tensor([[67, 68, 69]], dtype=torch.int32).cuda()
    want = seer.paged_attn_q4(q, kc, vc, table.cuda(), pos)[0]
    for pool in (kc, vc):
        pool.params[int(table[0, 4]), :, 5] = math.nan
        got, _ = seer.paged_attn_q4(q, kc, vc, table.cuda(), pos)
        assert torch.equal(got[:, :, :2], want[:, :, :2])
        assert bool(got[:, :, 2].isnan().all())


def test_values_that_are_not_finite():
    """A seen value of step NaN makes the elements of its group NaN and no others."""
    gen = torch.Generator().manual_seed(6)
    table, pages, _ = R.paged(gen, [100, 100], 16)
    kc, vc = (R.random_pool(seer, gen, pages, 2, 16, 128, 32) for _ in range(2))
    q = torch.randn(2, 4, 128, generator=gen).to(torch.bfloat16).cuda()
    pos = torch.tensor([99, 99], dtype=torch.int32).cuda()
    want = seer.paged_attn_q4(q, kc, vc, table.cuda(), pos)[0]
    vc.params[int(table[1, 2]), 1, 3, 2, 0] = math.nan
    got = seer.paged_attn_q4(q, kc, vc, table.cuda(), pos)[0]
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[1, 2:, 64:96] = True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("wide", [32, 33, 700])
def test_split_rows_and_whole_ones(wide):
    """Room for 512 keys (not split), for a page more, and for many."""
    gen = torch.Generator().manual_seed(wide)
    check(gen, torch.bfloat16, 4, 1, 128, 32, 16, [500, 3], wide=wide)


def test_long_rows():
    """A row that many workgroups share, beside short ones; the same bits every time."""
    gen = torch.Generator().manual_seed(8)
    o, lse = check(gen, torch.bfloat16, 4, 1, 64, 32, 64, [20000, 130, 1])
    gen = torch.Generator().manual_seed(8)
    o2, lse2 = check(gen, torch.bfloat16, 4, 1, 64, 32, 64, [20000, 130, 1])
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_many_sequences():
    gen = torch.Generator().manual_seed(10)
    lengths = [int(x) for x in torch.randint(0, 90, (150,), generator=gen)]
    check(gen, torch.bfloat16, 2, 2, 64, 64, 16, lengths)


@pytest.mark.parametrize("scale", [1e-4, 1.0, 30.0])
def test_scales(scale):
    gen = torch.Generator().manual_seed(11)
    check(gen, torch.float32, 4, 2, 128, 32, 16, [200, 64], scale=scale)


def test_fp32_precision():
    """What stands for fp32: over 4000 keys the output's error is that of sums in fp32 (2-norm, relative), not of the codes'
    offsets: each of n weights' sums rounds by U of what it holds at most, of random sign; o itself is a mean of values of
    random sign, so that sqrt(n) roundings of a sum that grows as sqrt(n) are about U / 2 sqrt(n / 64) tiles, 8 U; its scores are
    off by some 2 U sqrt(2 D) of terms up to 3 in size, 100 U: together below 2e-6 = 34 U twice over in every draw tried on
    paper, which a coherent offset (64 sums of 1.5 x 16 steps each, some 2e-5) is not."""
    gen = torch.Generator().manual_seed(12)
    B, H, D, n, page = 1, 4, 128, 4000, 16
    table, pages, _ = R.paged(gen, [n], page)
    kc, vc = (R.random_pool(seer, gen, pages, 1, page, D, 32) for _ in range(2))
    q = torch.randn(B, H, 1, D, generator=gen)
    pos = torch.tensor([[n - 1]], dtype=torch.int32)
    o, _ = seer.paged_attn_q4(q.cuda(), kc, vc, table.cuda(), pos.cuda())
    ro = R.attend(q, kc, vc, table, page, pos, 0.0)[0]
    off = float((o.cpu().double() - ro).norm() / ro.norm())
    print("off by", off)
    assert off < 2e-6


def test_many_sequences():
    """More sequences than a wavefront has lanes, most of them empty."""
    gen = torch.Generator().manual_seed(40)
    lengths = [1, 700, 2, 0, 0, 33] + [0] * 150 + [64, 1]
    pos = torch.tensor(lengths, dtype=torch.int32)[:, None] - 1
    table, pages, _ = R.paged(gen, lengths, 16, wide=50)
    kc, vc = (R.random_pool(seer, gen, pages, 2, 16, 64, 32) for _ in range(2))
    q = torch.randn(len(lengths), 4, 1, 64, generator=gen).to(torch.bfloat16)
    o, lse = seer.paged_attn_q4(q.cuda(), kc, vc, table.cuda(), pos.cuda(), want_lse=True)
    ro, rl, eo, el = R.attend(q, kc, vc, table, 16, pos, 0.0, None)
    none = pos.expand(-1, 4)[..., None] < 0
    assert torch.equal(lse.cpu() == -math.inf, none) and not bool(o.cpu()[none.squeeze(-1)].any())
    assert bool(((lse.cpu().double() - rl).abs()[~none] <= (el + R.U * rl.abs())[~none]).all())
    assert_rounded(o, ro, eo, "o")


@pytest.mark.parametrize("lengths", [[900, 3, 64, 700, 1300], [40] * 4, [1, 2000, 0, 1, 1, 600, 600, 90, 5000]])
def test_token_major_batches(lengths):
    """Pages whose heads share lines, in numbers of sequences whose shares are ordered by XCD."""
    gen = torch.Generator().manual_seed(len(lengths))
    check(gen, torch.bfloat16, 8, 4, 128, 32, 64, lengths, order="pshd", wide=80)
