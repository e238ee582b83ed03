"""Eviction (kv_evict) from rows that are longer than the registers of the workgroups that choose from them: such a workgroup reads its
weights again for each digit.  Equal weights, NaN and infinities lie on both sides of every border."""
import math
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

pytestmark = pytest.mark.gpu


def weights_of(gen, shape, kind):
    if kind == "few values":
        return torch.randint(0, 40, shape, generator=gen, device="cuda").float()
    w = torch.exp(2 * torch.randn(shape, generator=gen, device="cuda") - 6)
    if kind == "specials":
        at = torch.rand(shape, generator=gen, device="cuda")
        for i, x in enumerate((math.nan, math.inf, -math.inf, 0.0, -0.0, -1.0)):
            w[(at > 0.01 * i) & (at < 0.01 * i + 0.01)] = x
    return w


def want(w, n, keep, first, last):
    """Kept slots of a row [H, width] of length n > keep, by a stable sort (the lower of equal slots first): [H, keep]."""
    free = w[:, first:n - last].clone()
    free[free == 0] = 0.0
    top = free.nan_to_num(nan=math.inf, posinf=math.inf, neginf=-math.inf).sort(dim=1, descending=True, stable=True).indices
    # (NaN before infinity)
    isnan = free.isnan().gather(1, top)
    rank = isnan.to(torch.int8).sort(dim=1, descending=True, stable=True).indices
    top = top.gather(1, rank)[:, :keep - first - last] + first
    ends = torch.cat((torch.arange(first), n - last + torch.arange(last))).cuda().expand(w.shape[0], -1)
    return torch.cat((top, ends), 1).sort(dim=1).values


@pytest.mark.parametrize("kind", ["as they come", "few values", "specials"])
@pytest.mark.parametrize("B,H,room,lengths,keep,width", [
    # 130 rows, a workgroup each, of up to 40000 slots, some short
    (130, 1, 40000, [40000, 16385, 16384, 16383, 5, 0, 25001, 39999, 900], 700, 40000),
    (43, 3, 20011, [20011, 300, 17000], 6000, 18000),                          # (weights narrower than the rows)
    # 64 rows, four workgroups each, whose parts are longer than 16384 slots
    (32, 2, 90000, [90000, 66000, 65537, 70001, 40000, 100], 2048, 90000),
    # one row, 32 workgroups of 20000
    (1, 1, 640000, [640000], 5000, 640000),
])
def test_rows_longer_than_the_registers(kind, B, H, room, lengths, keep, width):
    page, first, last = 1024, 3, 17
    gen = torch.Generator(device="cuda").manual_seed(B + room)
    wide, need = -(-room // page), -(-keep // page)
    lengths = [lengths[b % len(lengths)] for b in range(B)]
    # the pool holds a sequence's pages once for all (they are only read), and the new ones
    pages = wide + B * need
    table = torch.arange(wide, dtype=torch.int32, device="cuda").expand(B, wide)
    to = (wide + torch.arange(B * need, dtype=torch.int32, device="cuda")).reshape(B, need)
    kc, vc = (torch.randint(0, 1 << 15, (pages, H, page, 64), generator=gen, device="cuda").to(torch.int16).view(torch.bfloat16)
              for _ in range(2))
    old = [kc[:wide].clone(), vc[:wide].clone()]
    w = weights_of(gen, (B, H, width), kind)
    n32 = torch.tensor(lengths, dtype=torch.int32).cuda()
    new_n, kept, new_w = seer.kv_evict(kc, vc, table, n32, w, to, keep, first=first, last=last)
    assert new_n.tolist() == [min(n, keep) for n in lengths]
    assert torch.equal(kc[:wide].view(torch.int16), old[0].view(torch.int16))
    for b, n in enumerate(lengths):
        rows = torch.nn.functional.pad(w[b], (0, max(n - width, 0)))
        m = min(n, keep)
        ref = want(rows, n, keep, first, last) if n > keep else torch.arange(n).cuda().expand(H, n)
        assert torch.equal(kept[b, :, :m].long(), ref) and bool((kept[b, :, m:] == -1).all())
        bits = rows.gather(1, ref).view(torch.int32)
        assert torch.equal(new_w[b, :, :m].view(torch.int32), bits) and not bool(new_w[b, :, m:].any())
        i, h = torch.arange(m).cuda(), torch.arange(H).cuda()[:, None]
        for a, x in zip(old, (kc, vc)):
            assert torch.equal(x[to[b].long()[i // page][None], h, (i % page)[None]].view(torch.int16),
                               a[ref // page, h, ref % page].view(torch.int16))
