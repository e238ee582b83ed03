"""Attention over a paged cache (seer_paged_attn) against softmax in 64 bits, within the bound of its
arithmetic (decode_ref.attend)."""
import math

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")

from decode_ref import assert_rounded, attend, freqs, make_cache, on_gpu  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN = float("nan")


def check(q, kc, vc, table, pos, order="phsd", scale=0.0, rope=None, **kw):
    """One call on the GPU against the reference; returns its outputs."""
    if rope is not None:
        kw.update(inv_freq=rope[0].cuda(), rope_scale=rope[1], interleaved=rope[2])
    o, lse = seer.paged_attn(q.cuda(), on_gpu(kc, order), on_gpu(vc, order), table.cuda(), pos.cuda(), sm_scale=scale,
                             want_lse=True, **kw)
    torch.cuda.synchronize()
    ro, rl, eo, el = attend(q, kc, vc, table, pos, scale, rope)
    assert_rounded(o.cpu(), ro, eo, "o")
    got = lse.cpu().double()
    empty = rl == -math.inf
    assert torch.equal(got == -math.inf, empty)
    assert bool(((got - rl).abs() <= el)[~empty].all()), float(((got - rl).abs() - el)[~empty].max())
    assert int(torch.count_nonzero(o.cpu()[empty])) == 0
    return o, lse


CASES = [
    # Hq, Hkv, D, tokens, page, order, rot, interleaved, lengths
    (2, 1, 64, 1, 16, "phsd", 0, False, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65]),
    (8, 2, 128, 1, 16, "phsd", 128, False, [127, 128, 129, 0, 511, 512, 513, 1000]),
    (28, 4, 128, 1, 1, "pshd", 0, False, [40, 3, 600, 0, 129]),
    (16, 16, 64, 1, 5, "phsd", 32, True, [700, 1, 64]),
    (40, 1, 128, 1, 24, "pshd", 48, False, [900, 31, 0, 1]),       # 40 rows: two blocks of 32
    (17, 1, 64, 1, 8, "phsd", 64, True, [513, 8]),
    (8, 2, 64, 3, 256, "pshd", 64, False, [3, 700, 257]),
    (28, 4, 128, 4, 64, "phsd", 0, False, [4, 1025, 100, 64]),
    (6, 2, 128, 7, 7, "phsd", 16, False, [7, 300, 66]),            # 21 rows
    (4, 4, 64, 33, 32, "pshd", 0, False, [33, 600]),               # three blocks of 16 rows
    (4, 2, 128, 1, 64, "phsd", 128, True, [20000, 300, 5000]),     # rows split over workgroups
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)).replace(" ", ""))
def test_matches_softmax(case, dtype):
    Hq, Hkv, D, S, ps, order, rot, inter, lengths = case
    print(f"[paged] {case} {dtype}", flush=True)
    gen = torch.Generator().manual_seed(sum(lengths) + D)
    # what no sequence holds is NaN
    kc, vc, table = make_cache(gen, lengths, ps, Hkv, D, TYPES[dtype], wide=-(-max(lengths) // ps) + 3, fill=NAN)
    q = (torch.randn(len(lengths), Hq, S, D, generator=gen) * 2).to(TYPES[dtype])
    pos = (torch.tensor(lengths)[:, None] - S + torch.arange(S)).to(torch.int32)
    check(q, kc, vc, table, pos, order, rope=(freqs(rot), 1.2, inter) if rot else None)
    check(q, kc, vc, table, pos, order, scale=0.3)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("ps", [3, 16])
def test_missing_pages_and_positions_beyond_the_table(dtype, ps):
    """Entries that are no page leave their keys out, also where that is every key; positions beyond the table see what
    it holds; negative ones see nothing."""
    gen = torch.Generator().manual_seed(11)
    lengths = [400, 400, 97, 300, 48]
    kc, vc, table = make_cache(gen, lengths, ps, 2, 64, TYPES[dtype], wide=-(-400 // ps), fill=NAN)
    pages = kc.shape[0]
    table[0, 1], table[0, 5], table[0, 6] = -1, pages, 2 ** 31 - 1
    table[1, :] = -7                      # nothing at all
    table[2, 0] = -2 ** 31                # the first page
    table[3, -(-300 // ps) - 1] = pages + 3  # the last one
    q = torch.randn(5, 6, 1, 64, generator=gen).to(TYPES[dtype])
    check(q, kc, vc, table, torch.tensor([[399], [399], [96], [299], [47]], dtype=torch.int32))
    cap = table.shape[1] * ps
    kc2, vc2, t2 = make_cache(gen, [cap] * 5, ps, 2, 64, TYPES[dtype])
    check(q, kc2, vc2, t2, torch.tensor([[cap], [2 ** 31 - 1], [cap - 1], [-1], [-2 ** 31]], dtype=torch.int32))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("G", [1, 5, 16])
def test_tokens_at_positions_of_their_own(dtype, G):
    """Padding among drafted tokens, tokens out of order, and tokens far apart."""
    gen = torch.Generator().manual_seed(G)
    lengths = [700, 130, 64, 900]
    kc, vc, table = make_cache(gen, lengths, 16, 2, 128, TYPES[dtype], fill=NAN)
    q = torch.randn(4, 2 * G, 4, 128, generator=gen).to(TYPES[dtype])
    pos = torch.tensor([[699, 698, -1, 697], [-1, -1, -1, 129], [0, 63, 62, 1], [3, 899, 450, -5]], dtype=torch.int32)
    check(q, kc, vc, table, pos, rope=(freqs(64), 1.0, False))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_unseen_values_of_later_tokens_do_not_reach_earlier_ones(dtype):
    """A drafted token whose K and V are NaN or infinite spoils its own row alone."""
    gen = torch.Generator().manual_seed(21)
    kc, vc, table = make_cache(gen, [330, 75], 16, 2, 64, TYPES[dtype], fill=NAN)
    q = torch.randn(2, 4, 3, 64, generator=gen).to(TYPES[dtype])
    pos = torch.tensor([[327, 328, 329], [72, 73, 74]], dtype=torch.int32)
    ref = attend(q, kc, vc, table, pos, 0.0)
    for bad in (NAN, math.inf, -math.inf):
        k2, v2 = kc.clone(), vc.clone()
        for b, p in ((0, 329), (1, 74)):
            k2[int(table[b, p // 16]), :, p % 16] = bad
            v2[int(table[b, p // 16]), :, p % 16] = bad
        o, lse = seer.paged_attn(q.cuda(), k2.cuda(), v2.cuda(), table.cuda(), pos.cuda(), want_lse=True)
        assert_rounded(o[:, :, :2].cpu(), ref[0][:, :, :2], ref[2][:, :, :2])
        assert bool(((lse[:, :, :2].cpu() - ref[1][:, :, :2]).abs() <= ref[3][:, :, :2]).all())
        assert not bool(torch.isfinite(o[:, :, 2]).all(-1).any())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_scores_beyond_the_finite(dtype):
    """As in the dense attention: +inf and NaN scores make their rows NaN, -inf is no weight, a row of nothing but -inf is empty;
    very large scores are ordinary ones."""
    gen = torch.Generator().manual_seed(31)
    n, D = 300, 64
    kc, vc, table = make_cache(gen, [n] * 5, 16, 1, D, TYPES[dtype])
    q = torch.zeros(5, 1, 1, D).to(TYPES[dtype])
    q[..., 0] = 8.0  # score = k[0] at head_dim 64
    at = lambda b, p: (int(table[b, p // 16]), 0, p % 16, 0)
    kc[..., 0] = kc[..., 0].clamp(-3, 3)
    kc[at(0, 100)] = math.inf
    kc[at(1, 299)] = NAN
    for p in range(0, 250):
        kc[at(2, p)] = -math.inf
    for p in range(n):
        kc[at(3, p)] = -math.inf
    kc[at(4, 17)] = 1e30
    pos = torch.full((5, 1), n - 1, dtype=torch.int32)
    o, lse = seer.paged_attn(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), pos.cuda(), want_lse=True)
    o, lse = o.cpu(), lse.cpu()
    assert bool(torch.isnan(o[:2]).all())
    assert int(torch.count_nonzero(o[3])) == 0 and lse[3].item() == -math.inf
    assert torch.equal(o[4, 0, 0], vc[at(4, 17)[0], 0, 17 % 16])
    few = torch.stack([kc[at(2, p)] for p in range(250, n)]).double()
    vals = torch.stack([vc[at(2, p)[0], 0, p % 16] for p in range(250, n)]).double()
    p = torch.softmax(few, 0)
    # scores are at most 3: (D + 2) u 3 + 4 u 4 each, as in decode_ref
    e = 2 * ((D + 2) * 3 + 16) * 2.0 ** -24 + 2 * 308 * 2.0 ** -24 + 2.0 ** -16
    assert_rounded(o[2, 0, 0], p @ vals, e * (p @ vals.abs()))


def test_many_ragged_sequences_and_padding_rows():
    """More sequences than a workgroup has threads, most of them short, some of them empty."""
    gen = torch.Generator().manual_seed(41)
    lengths = [int(x) for x in torch.randint(0, 40, (600,), generator=gen)]
    lengths[5], lengths[300], lengths[599] = 3000, 1500, 900
    kc, vc, table = make_cache(gen, lengths, 16, 1, 64, torch.bfloat16, fill=NAN)
    q = torch.randn(600, 2, 1, 64, generator=gen).bfloat16()
    pos = (torch.tensor(lengths) - 1).to(torch.int32)[:, None]
    o, lse = check(q, kc, vc, table, pos)
    # [B, H, D] queries with [B] positions are the same call, and it gives the same bits
    o2, l2 = seer.paged_attn(q[:, :, 0].cuda(), kc.cuda(), vc.cuda(), table.cuda(), pos[:, 0].contiguous().cuda(), want_lse=True)
    assert torch.equal(o2, o[:, :, 0]) and torch.equal(l2, lse[:, :, 0])


def test_shared_pages_and_repeated_rows():
    """Two sequences on the same pages (a shared prompt), and the same result on every run."""
    gen = torch.Generator().manual_seed(51)
    kc, vc, table = make_cache(gen, [5000], 64, 2, 128, torch.bfloat16)
    table = table.expand(7, -1).contiguous()
    q = torch.randn(1, 8, 1, 128, generator=gen).bfloat16().expand(7, 8, 1, 128).contiguous()
    pos = torch.tensor([[4999], [4999], [2000], [10], [4999], [63], [64]], dtype=torch.int32)
    o, lse = check(q, kc, vc, table, pos)
    for _ in range(3):
        o2, l2 = seer.paged_attn(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), pos.cuda(), want_lse=True)
        assert torch.equal(o, o2) and torch.equal(lse, l2)


def test_strided_operands_and_untouched_surroundings():
    """q, o and the table as parts of larger buffers; a workspace full of NaN; nothing else is written."""
    gen = torch.Generator().manual_seed(61)
    lengths = [2500, 77, 0]
    kc, vc, table = make_cache(gen, lengths, 16, 2, 128, torch.bfloat16, fill=NAN)
    wide = torch.full((3, table.shape[1] + 9), -1, dtype=torch.int32)
    wide[:, 4:4 + table.shape[1]] = table
    big = torch.randn(3, 2, 14, 128, generator=gen).bfloat16()
    q = big[:, :, 3:11].transpose(1, 2)  # [3, 8, 2, 128], token-major
    pos = torch.tensor([[2498, 2499], [75, 76], [-1, -1]], dtype=torch.int32)
    out = torch.full((3, 2, 14, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    gq = big.cuda()[:, :, 3:11].transpose(1, 2)
    need = seer.paged_attn_workspace_bytes(gq, kc.cuda(), vc.cuda(), table.cuda())
    ws = torch.full((need // 4 + 64,), NAN, device="cuda")
    o, lse = seer.paged_attn(gq, kc.cuda(), vc.cuda(), wide.cuda()[:, 4:4 + table.shape[1]], pos.cuda(),
                             out=out[:, :, 3:11].transpose(1, 2), want_lse=True, workspace=ws)
    ref = attend(q, kc, vc, table, pos, 0.0)
    assert_rounded(o.cpu(), ref[0], ref[2])
    assert bool((out[:, :, :3] == 9).all()) and bool((out[:, :, 11:] == 9).all())
    assert bool(torch.isnan(ws[need // 4:]).all())


def test_cache_of_more_than_32_bits_of_elements():
    H, ps, D, n = 2, 512, 128, 1300
    pages = (1 << 32) // (H * ps * D) + 8
    print("[paged] long cache", flush=True)
    gen = torch.Generator().manual_seed(71)
    kc, vc = (torch.empty(pages, H, ps, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k3, v3 = (torch.randn(3, H, ps, D, generator=gen).bfloat16() for _ in range(2))
    where = [pages - 1, 0, pages - 4]
    for i, p in enumerate(where):
        kc[p], vc[p] = k3[i].cuda(), v3[i].cuda()
    table = torch.tensor([where], dtype=torch.int32)
    q = torch.randn(1, 8, 1, D, generator=gen).bfloat16()
    pos = torch.tensor([[n - 1]], dtype=torch.int32)
    o, lse = seer.paged_attn(q.cuda(), kc, vc, table.cuda(), pos.cuda(), want_lse=True)
    ref = attend(q, k3, v3, torch.tensor([[0, 1, 2]], dtype=torch.int32), pos, 0.0)
    assert_rounded(o.cpu(), ref[0], ref[2])
    assert bool(((lse.cpu() - ref[1]).abs() <= ref[3]).all())


def test_layouts_are_checked():
    q = torch.zeros(2, 4, 1, 64, device="cuda")
    kc = torch.zeros(4, 2, 8, 64, device="cuda")
    table = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    pos = torch.zeros(2, 1, dtype=torch.int32, device="cuda")

    def call(q=q, kc=kc, vc=kc, table=table, pos=pos, **kw):
        return seer.paged_attn(q, kc, vc, table, pos, **kw)

    call()
    assert call(q=q[:0], table=table[:0], pos=pos[:0])[0].shape == (0, 4, 1, 64)
    for bad in (dict(q=q[0, 0]), dict(table=table[:1]), dict(pos=pos[:1]), dict(pos=torch.cat([pos, pos], 1)), dict(vc=kc[:2]),
                dict(kc=kc[..., :32], vc=kc[..., :32]), dict(out=q[:1]), dict(q=q.cpu()), dict(table=table.cpu()),
                dict(workspace=torch.zeros(1 << 24)), dict(lse=torch.zeros(2, 4, 2, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(q=q.bfloat16()), dict(pos=pos.long()), dict(q=q.half(), kc=kc.half(), vc=kc.half())):
        with pytest.raises(TypeError):
            call(**bad)
    with pytest.raises(seer.SeerError) as e:
        call(q=torch.zeros(2, 5, 1, 64, device="cuda"))
    assert e.value.status == seer.ERR_INVALID_ARG
    with pytest.raises(seer.SeerError) as e:
        call(workspace=torch.zeros(100, device="cuda"))
    assert e.value.status == seer.ERR_WORKSPACE
