"""Attention weights of cached keys (kv_weights) whose scores are large: a key's weight is as exact as its distance from the row's
log-sum-exp is small, however large both are."""
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [1, 9])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,kind", [(torch.bfloat16, "q4"), (torch.float32, "q4"), (torch.bfloat16, "bf16"), (torch.float32, "f32")])
def test_large_scores(dtype, kind, D, S):
    """A row has one element, 16, in a group's first channel, where keys hold 18 + (c - 7.5) / 16: scores of 280.5 to 295.5, exact in fp32,
    against log-sum-exps of 288 to 292.  With x the difference, a term is then off by the roundings of x, of log2(e) and their product,
    (1 + 1 / 4 + 1) U |x|, and of the power, one unit in the last place, 2 U: less than (2.5 |x| + 3) U of it; and a key's sum by
    U for each of its rows."""
    gen = torch.Generator().manual_seed(D + S)
    Hq, Hkv, page, lengths = 4, 2, 16, [200, 70]
    table, pages, _ = R.paged(gen, lengths, page)
    c = torch.randint(0, 16, (pages, Hkv, page, D), generator=gen)
    if kind == "q4":
        params = torch.empty(pages, Hkv, page, D // 32, 2)
        params[..., 0], params[..., 1] = 2.0 ** -4, 18.0
        kc = seer.Q4Pool((c[..., 0::2] | c[..., 1::2] << 4).to(torch.uint8).cuda(), params.to(torch.bfloat16).cuda())
    else:
        # (bf16 holds eighths of 18)
        kc = (18 + (c - 7.5).div(2, rounding_mode="floor") / 8).to(dtype).cuda()
    q = torch.zeros(2, Hq, S, D, dtype=dtype)
    q[..., 32] = 16.0
    pos = (torch.tensor(lengths)[:, None] - S + torch.arange(S)).to(torch.int32)
    lse = 288.0 + 4.0 * torch.rand(2, Hq, S, generator=gen)
    w = torch.zeros(2, Hkv, table.shape[1] * page).cuda()
    seer.kv_weights(q.cuda(), kc, table.cuda(), pos.cuda(), lse.cuda(), w, decay=0.0, sm_scale=1.0)
    k = R.values(kc)
    for b, n in enumerate(lengths):
        kb = R.rows_of(k, table[b], page, n)
        for g in range(Hkv):
            ref, bound = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
            for s in range(S):
                seen = R.seen_of(table[b], page, pages, int(pos[b, s]), n)
                for h in range(2 * g, 2 * g + 2):
                    x = 16.0 * kb[:, g, 32] - float(lse[b, h, s])
                    p = torch.where(seen, torch.exp(x), 0.0)
                    ref += p
                    bound += p * (2.5 * x.abs() + 3) * R.U
            bound += 2 * S * R.U * ref
            d = (w[b, g, :n].cpu().double() - ref).abs()
            assert bool((d <= bound).all()), float((d / ref.clamp_min(1e-300)).max())
