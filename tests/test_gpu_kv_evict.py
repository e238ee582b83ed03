"""Eviction by weight (kv_evict): which slots stay is exact, and keys and values are moved as they are."""
import math
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

import cache_ref as R  # noqa: E402

pytestmark = pytest.mark.gpu


def planes(pool):
    """A pool's tensors as bytes, [pages, heads, slots, ..] (CPU copies)."""
    ts = (pool.codes, pool.params) if hasattr(pool, "codes") else (pool,)
    return [t.cpu().contiguous().view(torch.uint8).clone() for t in ts]


def check(gen, kind, H, D, group, page, lengths, keep, first, last, weights=None, width=None, order="phsd", wide=None, hole=None,
          slack=0):
    B = len(lengths)
    need = -(-keep // page) + slack
    table, pages, free = R.paged(gen, lengths, page, spare=B * need + 1, wide=wide)
    to = torch.tensor(free[:B * need], dtype=torch.int32).reshape(B, need)
    if kind == "q4":
        kc, vc = (R.random_pool(seer, gen, pages, H, page, D, group, order) for _ in range(2))
    else:
        dt = torch.bfloat16 if kind == "bf16" else torch.float32
        kc, vc = (torch.randn(pages, page, H, D, generator=gen).to(dt).cuda().transpose(1, 2) if order == "pshd" else
                  torch.randn(pages, H, page, D, generator=gen).to(dt).cuda() for _ in range(2))
    if hole is not None:
        table[hole] = -1
    cap = table.shape[1] * page
    W = cap if width is None else width
    w = torch.rand(B, H, W, generator=gen) if weights is None else weights
    old = [planes(kc), planes(vc)]
    n32 = torch.tensor(lengths, dtype=torch.int32).cuda()
    new_n, kept, new_w = seer.kv_evict(kc, vc, table.cuda(), n32, w.cuda(), to.cuda(), keep, first=first, last=last)
    want = R.evict(w, lengths, keep, first, last, cap)
    assert new_n.tolist() == [len(x[0]) for x in want]
    assert new_w.shape[2] == need * page
    for x, now in zip(old, (planes(kc), planes(vc))):
        for a in x:  # what the definition makes of the old bytes
            ref = a.clone()
            for b in range(B):
                for h in range(H):
                    for i, s in enumerate(want[b][h]):
                        p = int(table[b, s // page])
                        if 0 <= p < pages:
                            ref[int(to[b, i // page]), h, i % page] = a[p, h, s % page]
            a.copy_(ref)
        for a, c in zip(x, now):
            assert torch.equal(a, c)
    for b in range(B):
        for h in range(H):
            ks = want[b][h]
            assert kept[b, h].tolist() == ks + [-1] * (keep - len(ks))
            ref = torch.zeros(need * page)
            for i, s in enumerate(ks):
                ref[i] = w[b, h, s] if s < W else 0.0
            assert torch.equal(new_w[b, h].cpu().nan_to_num(7.0), ref.nan_to_num(7.0))


@pytest.mark.parametrize("kind,H,D,group", [("bf16", 2, 128, 0), ("bf16", 1, 64, 0), ("f32", 2, 64, 0), ("f32", 1, 128, 0), ("q4", 2, 128, 32),
                                            ("q4", 2, 128, 64), ("q4", 3, 64, 32), ("q4", 1, 64, 64)])
@pytest.mark.parametrize("order", ["phsd", "pshd"])
def test_kinds_of_cache(kind, H, D, group, order):
    gen = torch.Generator().manual_seed(D + group)
    check(gen, kind, H, D, group, 16, [100, 0, 33, 32, 1, 70], 32, 4, 8, order=order)


@pytest.mark.parametrize("page", [1, 3, 24, 64])
@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (1, 1, 0), (2, 1, 1), (10, 0, 10), (10, 10, 0), (17, 3, 5), (100, 2, 30)])
def test_budgets(page, keep, first, last):
    gen = torch.Generator().manual_seed(keep + page)
    check(gen, "bf16", 2, 64, 0, page, [101, 100, 99, 18, 17, 2, 1], keep, first, last)


def test_equal_weights_keep_the_lower_slots():
    gen = torch.Generator().manual_seed(1)
    w = torch.randint(0, 4, (3, 2, 2000), generator=gen).float()
    w[1] = 0.5
    w[2, 0, ::2], w[2, 0, 1::2] = 0.0, -0.0
    check(gen, "q4", 2, 64, 32, 16, [2000, 1500, 1999], 700, 5, 9, weights=w)


def test_weights_of_all_kinds():
    """Negative, tiny, infinite and NaN weights have their order."""
    gen = torch.Generator().manual_seed(2)
    w = torch.randn(2, 1, 320, generator=gen) * torch.exp(30 * torch.randn(2, 1, 320, generator=gen))
    w[0, 0, 10], w[0, 0, 20], w[0, 0, 30:60] = math.inf, -math.inf, 1e-42
    w[1, 0, 5], w[1, 0, 6], w[1, 0, 7] = math.nan, -math.nan, math.inf
    w.view(torch.int32)[1, 0, 9] = -4194303  # (a NaN with its sign bit)
    for keep in (1, 3, 150):
        check(gen, "bf16", 1, 64, 0, 16, [320, 320], keep, 0, 0, weights=w)


@pytest.mark.parametrize("n", [1023, 1024, 1025, 5000, 20000])
def test_long_rows(n):
    """Lengths around the workgroup's, with weights as they come (a few have most)."""
    gen = torch.Generator().manual_seed(n)
    w = torch.exp(2 * torch.randn(1, 1, n + 7, generator=gen) - 6)
    check(gen, "q4", 1, 64, 64, 64, [n], n // 3, 4, 16, weights=w, width=n + 7)


@pytest.mark.parametrize("ties", [False, True])
def test_rows_in_parts(ties):
    """Rows of several workgroups: the weight that decides has equals in all parts, or every slot has the same."""
    gen = torch.Generator().manual_seed(11)
    w = torch.randint(0, 50, (2, 2, 50000), generator=gen).float() if not ties else torch.ones(2, 2, 50000)
    check(gen, "q4", 2, 64, 64, 64, [50000, 17000], 20011, 3, 40, weights=w, width=50000)


def test_weights_narrower_than_the_rows():
    """Slots beyond the weights weigh 0."""
    gen = torch.Generator().manual_seed(4)
    check(gen, "bf16", 2, 64, 0, 16, [90, 200], 60, 0, 5, width=50)


def test_lengths_out_of_range_and_holes():
    """A negative length is 0, one beyond the table what it has room for; a slot without a page is not moved; room behind the
    kept slots is left."""
    gen = torch.Generator().manual_seed(5)
    check(gen, "f32", 1, 64, 0, 8, [40, 64], 20, 2, 3, hole=(1, 2), slack=2)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32).cuda()
    to = torch.tensor([[4], [5]], dtype=torch.int32).cuda()
    kc, vc = (torch.randn(6, 1, 8, 64, generator=gen).cuda() for _ in range(2))
    w = torch.rand(2, 1, 16, generator=gen).cuda()
    n, kept, _ = seer.kv_evict(kc, vc, table, torch.tensor([-5, 1000], dtype=torch.int32).cuda(), w, to, 6, last=2)
    assert n.tolist() == [0, 6] and kept[0, 0].tolist() == [-1] * 6
    assert kept[1, 0].tolist() == R.evict(w.cpu(), [0, 16], 6, 0, 2, 16)[1][0]
    assert torch.equal(kc[5, 0, :6], torch.cat((kc[2, 0], kc[3, 0]))[kept[1, 0].long()])


@pytest.mark.parametrize("n", [300, 40000])
def test_lengths_in_place(n):
    """New lengths over the old ones, short rows (a workgroup each) and long ones (several)."""
    gen = torch.Generator().manual_seed(n)
    table, pages, free = R.paged(gen, [n, n, n], 64, spare=6)
    to = torch.tensor(free[:6], dtype=torch.int32).reshape(3, 2).cuda()
    kc, vc = (torch.randn(pages, 2, 64, 64, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    w = torch.rand(3, 2, n, generator=gen)
    lengths = [n, 90, n - 1]
    n32 = torch.tensor(lengths, dtype=torch.int32).cuda()
    out = (n32, torch.empty(3, 2, 100, dtype=torch.int32).cuda(), torch.empty(3, 2, 100).cuda())
    back, kept, _ = seer.kv_evict(kc, vc, table.cuda(), n32, w.cuda(), to, 100, first=2, last=5, out=out)
    assert back is n32 and n32.tolist() == [100, 90, 100]
    for b, x in enumerate(R.evict(w, lengths, 100, 2, 5, table.shape[1] * 64)):
        for h in range(2):
            assert kept[b, h].tolist() == x[h] + [-1] * (100 - len(x[h]))


@pytest.mark.parametrize("kind,B,keep", [("bf16", 4, 4200), ("q4", 8, 8200)])
def test_large_moves(kind, B, keep):
    """More than the caches hold."""
    gen = torch.Generator().manual_seed(B)
    H, page, n = 8, 64, keep + 100
    table, pages, free = R.paged(gen, [n] * B, page, spare=B * (-(-keep // page)))
    table, to = table.cuda(), torch.tensor(free, dtype=torch.int32)[:B * (-(-keep // page))].reshape(B, -1).cuda()
    if kind == "q4":
        kc, vc = seer.alloc_kv_cache_q4(pages, page, H, 128)
        for p in (kc, vc):
            p.codes.random_(0, 256)
            p.params.copy_(torch.rand(p.params.shape, device="cuda"))
        planes_of = (kc.codes, kc.params, vc.codes, vc.params)
    else:
        kc, vc = planes_of = [torch.rand(pages, H, page, 128, device="cuda").to(torch.bfloat16) for _ in range(2)]
    w = torch.rand(B, H, n, generator=gen).cuda()
    old = [p.clone() for p in planes_of]
    n32 = torch.full((B,), n, dtype=torch.int32).cuda()
    _, kept, new_w = seer.kv_evict(kc, vc, table, n32, w, to, keep)
    want = w.sort(dim=2, descending=True, stable=True).indices[..., :keep].sort(dim=2).values  # (of equal ones the lower slot)
    assert torch.equal(kept.long(), want)
    assert torch.equal(new_w[:, :, :keep], w.gather(2, want))
    i, h = torch.arange(keep).cuda(), torch.arange(H).cuda()[None, :, None]
    src = table.long().gather(1, (want // page).reshape(B, -1)).reshape(B, H, keep)
    dst = to.long()[:, i // page][:, None].expand(B, H, keep)
    for a, p in zip(old, planes_of):
        assert torch.equal(p[dst, h, i % page], a[src, h, want % page])
