"""Attention over a cache in 4 bits in the mean (2-norms), for every form of the kernel: what the header states (q whole, weights whole or
in two parts, codes that are centred where the output is fp32) leaves no more than the roundings that it names."""
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402
import cache_tight as T  # noqa: E402
from decode_ref import freqs  # noqa: E402
from test_gpu_q4_attn import SHAPES, check as check_elements  # noqa: E402

pytestmark = pytest.mark.gpu


def check(gen, dtype, Hq, Hkv, D, group, page, lengths, S=1, turn=None, pool=T.random_pool, wide=None):
    table, pages, _ = R.paged(gen, lengths, page, wide=wide)
    kc, vc = (pool(seer, gen, pages, Hkv, page, D, group) for _ in range(2))
    q = (1.5 * torch.randn(len(lengths), Hq, S, D, generator=gen)).to(dtype)
    pos = (torch.tensor(lengths)[:, None] - S + torch.arange(S)).to(torch.int32)
    how = {} if turn is None else dict(inv_freq=turn[0].cuda(), rope_scale=turn[1], interleaved=turn[2])
    o, lse = seer.paged_attn_q4(q.cuda(), kc, vc, table.cuda(), pos.cuda(), want_lse=True, **how)
    T.check(o, lse, T.attend(q, kc, vc, table, page, pos, 0.0, turn), f"{dtype} {Hq} / {Hkv} x {D}, groups of {group}:")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("lengths", [[1, 2, 1, 3], [70, 300]])
@pytest.mark.parametrize("Hq,Hkv,D,group", SHAPES)
def test_forms(dtype, rotated, lengths, Hq, Hkv, D, group):
    """Rows of one key have their score as their log-sum-exp, where a part of q left out shows; longer ones show the weights'."""
    gen = torch.Generator().manual_seed(Hq + D + group + len(lengths))
    check(gen, dtype, Hq, Hkv, D, group, 16, lengths, turn=(freqs(D, 500000.0), 1.1, False) if rotated else None, wide=40)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S,Hq,Hkv,D,group", [(3, 8, 2, 128, 32), (4, 7, 1, 128, 64), (2, 8, 1, 64, 32), (9, 2, 1, 64, 64)])
def test_several_tokens(dtype, S, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(S)
    check(gen, dtype, Hq, Hkv, D, group, 24, [90, 130], S=S, turn=(freqs(D // 2, 10000.0), 1.0, True))


@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,group", SHAPES)
def test_codes_of_fp32_are_centred(rotated, Hq, Hkv, D, group):
    """Elements near their group's middle, with one far off in each group: codes that enter as 1 + c / 16 carry the rounding of
    numbers some fifteen times the values'."""
    gen = torch.Generator().manual_seed(Hq + D + group + 3)
    check(gen, torch.float32, Hq, Hkv, D, group, 16, [70, 300], turn=(freqs(D, 500000.0), 1.0, False) if rotated else None,
          pool=T.outlier_pool)


def test_fp32_over_many_keys():
    gen = torch.Generator().manual_seed(21)
    check(gen, torch.float32, 4, 1, 128, 32, 16, [4000])
    check(gen, torch.float32, 4, 1, 64, 64, 16, [1000], pool=T.outlier_pool)


def test_many_sequences_of_single_groups():
    """150 sequences of up to 90 keys, several to a lane; a head is a group, and each query head has its own."""
    gen = torch.Generator().manual_seed(10)
    lengths = [int(x) for x in torch.randint(0, 90, (150,), generator=gen)]
    check_elements(gen, torch.bfloat16, 2, 2, 64, 64, 16, lengths)
