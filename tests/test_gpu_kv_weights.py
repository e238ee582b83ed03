"""The attention weights of cached keys (kv_weights) against the definition in 64 bits."""
import math
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402
from decode_ref import freqs  # noqa: E402

pytestmark = pytest.mark.gpu


def pool(gen, pages, H, page, D, kind, group, order="phsd"):
    if kind == "q4":
        return R.random_pool(seer, gen, pages, H, page, D, group, order)
    dt = torch.bfloat16 if kind == "bf16" else torch.float32
    x = torch.randn(pages, H, page, D, generator=gen).to(dt)
    return x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if order == "pshd" else x.cuda()


def check(gen, dtype, Hq, Hkv, D, group, page, lengths, S=1, kind="q4", order="phsd", decay=1.0, turn=None, wide=None, width=None,
          pos=None, lse=None, mend=None, scale=0.0):
    B = len(lengths)
    table, pages, _ = R.paged(gen, lengths, page, wide=wide)
    kc = pool(gen, pages, Hkv, page, D, kind, group, order)
    q = (1.5 * torch.randn(B, Hq, S, D, generator=gen)).to(dtype)
    if pos is None:
        pos = (torch.tensor(lengths)[:, None] - S + torch.arange(S)).to(torch.int32)
    if lse is None:
        lse = 3.0 + torch.rand(B, Hq, S, generator=gen)
    if mend is not None:
        mend(kc, table)
    W = table.shape[1] * page if width is None else width
    w0 = torch.rand(B, Hkv, W, generator=gen)
    how = {} if turn is None else dict(inv_freq=turn[0].cuda(), rope_scale=turn[1], interleaved=turn[2])
    ref, err = R.weigh(q, kc, table, page, pos, lse, w0, decay, scale, W, turn)
    got = w0.clone() if decay else torch.where(err > 0, math.nan, w0.double()).float()  # (what is not read may be anything)
    got = got.cuda()
    back = seer.kv_weights(q.cuda(), kc, table.cuda(), pos.cuda(), lse.cuda(), got, decay=decay, sm_scale=scale, **how)
    assert back is got
    d = (got.cpu().double() - ref).abs()
    assert bool((d <= err).all()), float((d - err).max())
    return got


@pytest.mark.parametrize("dtype,kind", [(torch.bfloat16, "q4"), (torch.float32, "q4"), (torch.bfloat16, "bf16"), (torch.float32, "f32")])
@pytest.mark.parametrize("Hq,Hkv,D,group", [(2, 1, 64, 32), (2, 1, 64, 64), (12, 12, 64, 32), (8, 2, 128, 32), (8, 2, 128, 64),
                                            (7, 1, 128, 32), (24, 1, 128, 64)])
def test_one_token(dtype, kind, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(Hq + D + group)
    check(gen, dtype, Hq, Hkv, D, group, 16, [1, 63, 64, 65, 300], kind=kind, wide=20)


@pytest.mark.parametrize("dtype,kind", [(torch.bfloat16, "q4"), (torch.float32, "q4"), (torch.bfloat16, "bf16"), (torch.float32, "f32")])
@pytest.mark.parametrize("S,Hq,Hkv,D,group", [(2, 4, 2, 64, 32), (33, 4, 1, 128, 32), (64, 2, 2, 64, 64), (5, 14, 2, 128, 64)])
def test_windows_rotated(dtype, kind, S, Hq, Hkv, D, group):
    """Several tokens, which see different keys; more rows than the LDS holds at a time; keys decayed."""
    gen = torch.Generator().manual_seed(S)
    check(gen, dtype, Hq, Hkv, D, group, 24, [S + 130, S, 66], S=S, kind=kind, order="pshd", decay=0.75,
          turn=(freqs(D // 2, 500000.0), 1.1, True))


@pytest.mark.parametrize("kind", ["q4", "bf16", "f32"])
@pytest.mark.parametrize("page", [1, 5, 8, 16, 100])
def test_page_sizes_and_fresh_weights(kind, page):
    gen = torch.Generator().manual_seed(page)
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    check(gen, dtype, 4, 2, 128, 32, page, [200, 7, 131], S=9, kind=kind, decay=0.0)


@pytest.mark.parametrize("kind", ["q4", "bf16", "f32"])
def test_rows_without_keys(kind):
    """Rows of lse -inf count nothing; unseen slots and pages that do not exist may hold anything; sequences without tokens,
    many of them, leave their weights."""
    gen = torch.Generator().manual_seed(2)
    lengths = [0, 0, 0, 40, 33, 0, 50, 20] + [0] * 140 + [30]
    B = len(lengths)
    pos = torch.stack([torch.tensor([n - 2, n - 1]) if n else torch.tensor([-1, -3]) for n in lengths]).to(torch.int32)
    lse = 3.0 + torch.rand(B, 4, 2, generator=gen)
    lse[3, 1] = -math.inf
    lse[6, :, 0] = -math.inf

    def mend(kc, table):
        table[4] = -1
        table[6, 0] = 10 ** 6
        params = kc.params if kind == "q4" else kc
        real = torch.zeros(params.shape[0], params.shape[2], dtype=torch.bool)
        for b, n in enumerate(lengths):
            for t in range(n):
                p = int(table[b, t // 16])
                if 0 <= p < real.shape[0]:
                    real[p, t % 16] = True
        real = real[:, None, :].reshape(real.shape[0], 1, real.shape[1], *[1] * (params.dim() - 3))
        params.copy_(torch.where(real.cuda(), params, math.nan))

    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    # (the reference multiplies what it masks: NaN there stays out of it by where)
    check(gen, dtype, 4, 2, 64, 32, 16, lengths, S=2, kind=kind, wide=6, pos=pos, lse=lse, mend=mend)


@pytest.mark.parametrize("width", [1, 50, 64, 131])
def test_keys_beyond_the_weights(width):
    gen = torch.Generator().manual_seed(width)
    check(gen, torch.bfloat16, 4, 2, 128, 32, 16, [130, 20], width=width)


@pytest.mark.parametrize("kind", ["q4", "bf16"])
def test_long_rows_and_bits(kind):
    gen = torch.Generator().manual_seed(8)
    a = check(gen, torch.bfloat16, 4, 1, 64, 32, 64, [9000, 130, 1], kind=kind)
    gen = torch.Generator().manual_seed(8)
    assert torch.equal(a, check(gen, torch.bfloat16, 4, 1, 64, 32, 64, [9000, 130, 1], kind=kind))


def test_another_output():
    """out: weights stay, what is not counted stays in out, strides differ."""
    gen = torch.Generator().manual_seed(3)
    table, pages, _ = R.paged(gen, [40], 16)
    kc = R.random_pool(seer, gen, pages, 2, 16, 64, 32)
    q = torch.randn(1, 4, 64, generator=gen).cuda()
    pos, lse = torch.tensor([39], dtype=torch.int32).cuda(), torch.full((1, 4), 4.0).cuda()
    w = torch.rand(1, 2, 48, generator=gen).cuda()
    keep = w.clone()
    out = torch.full((1, 2, 100), 5.0).cuda()[:, :, :48]
    seer.kv_weights(q, kc, table.cuda(), pos, lse, w, out=out)
    assert torch.equal(w, keep) and bool((out[:, :, 40:] == 5.0).all())
    seer.kv_weights(q, kc, table.cuda(), pos, lse, w)
    assert torch.equal(out[:, :, :40], w[:, :, :40])


@pytest.mark.parametrize("kind", ["q4", "bf16"])
def test_weights_sum_to_the_rows(kind):
    """With the lse of the attention call the weights of a sequence's keys add up to its rows: each within its lse's error (some
    1e-5) of 1."""
    gen = torch.Generator().manual_seed(5)
    lengths = [300, 20]
    table, pages, _ = R.paged(gen, lengths, 16)
    kc = pool(gen, pages, 2, 16, 128, kind, 32)
    q = torch.randn(2, 8, 3, 128, generator=gen).to(torch.bfloat16).cuda()
    pos = (torch.tensor(lengths)[:, None] - 3 + torch.arange(3)).to(torch.int32).cuda()
    f = freqs(128).cuda()
    attn = seer.paged_attn_q4 if kind == "q4" else seer.paged_attn
    lse = attn(q, kc, kc, table.cuda(), pos, inv_freq=f, want_lse=True)[1]
    w = torch.zeros(2, 2, table.shape[1] * 16).cuda()
    seer.kv_weights(q, kc, table.cuda(), pos, lse, w, inv_freq=f)
    assert bool(((w.sum(-1) - 12).abs() < 12 * 2e-5).all())


@pytest.mark.parametrize("kind", ["q4", "bf16"])
@pytest.mark.parametrize("lengths", [[900, 3, 64, 700, 1300], [40] * 4, [1, 2000, 0, 1, 1, 600, 600, 90, 5000]])
def test_token_major_batches(kind, lengths):
    """Pages whose heads share lines, in numbers of sequences whose shares are ordered by XCD."""
    gen = torch.Generator().manual_seed(len(lengths))
    check(gen, torch.bfloat16, 8, 4, 128, 32, 64, lengths, kind=kind, order="pshd", wide=80)
