"""The attention weights of cached keys (kv_weights) in the mean (2-norms), over a cache in 4 bits."""
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402
import cache_tight as T  # noqa: E402
from decode_ref import freqs  # noqa: E402

pytestmark = pytest.mark.gpu
SHAPES = [(2, 1, 64, 32), (2, 1, 64, 64), (12, 12, 64, 32), (8, 2, 128, 32), (8, 2, 128, 64), (7, 1, 128, 32), (24, 1, 128, 64)]


def check(gen, dtype, Hq, Hkv, D, group, page, lengths, S=1, turn=None, pool=T.random_pool):
    table, pages, _ = R.paged(gen, lengths, page)
    kc = pool(seer, gen, pages, Hkv, page, D, group)
    q = (1.5 * torch.randn(len(lengths), Hq, S, D, generator=gen)).to(dtype)
    pos = (torch.tensor(lengths)[:, None] - S + torch.arange(S)).to(torch.int32)
    lse = T.attend(q, kc, kc, table, page, pos, 0.0, turn)[1].float()
    how = {} if turn is None else dict(inv_freq=turn[0].cuda(), rope_scale=turn[1], interleaved=turn[2])
    w = torch.zeros(len(lengths), Hkv, table.shape[1] * page).cuda()
    seer.kv_weights(q.cuda(), kc, table.cuda(), pos.cuda(), lse.cuda(), w, decay=0.0, **how)
    ref, err = T.weigh(q, kc, table, page, pos, lse, 0.0, turn)
    off = T.norm(w.cpu().double() - ref)
    print(f"{dtype} {Hq} / {Hkv} x {D}, groups of {group}: {off / T.norm(ref):.2e} (allowed {T.MARGIN * T.norm(err) / T.norm(ref):.2e})")
    assert off <= T.MARGIN * T.norm(err)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,group", SHAPES)
def test_forms(dtype, rotated, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(Hq + D + group)
    check(gen, dtype, Hq, Hkv, D, group, 16, [5, 70, 300], turn=(freqs(D, 500000.0), 1.1, False) if rotated else None)


@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,group", SHAPES)
def test_codes_of_fp32_are_centred(rotated, Hq, Hkv, D, group):
    """Elements near their group's middle, with one far off in each group: codes that enter as 1 + c / 16 carry the rounding of
    numbers some fifteen times the values'."""
    gen = torch.Generator().manual_seed(Hq + D + group + 3)
    check(gen, torch.float32, Hq, Hkv, D, group, 16, [70, 300], turn=(freqs(D, 500000.0), 1.0, False) if rotated else None,
          pool=T.outlier_pool)


def test_windows_of_fp32():
    gen = torch.Generator().manual_seed(33)
    check(gen, torch.float32, 8, 2, 128, 32, 24, [200, 40], S=33, turn=(freqs(64, 500000.0), 1.0, True), pool=T.outlier_pool)
