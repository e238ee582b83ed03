"""The append of new keys and values to a paged cache (seer_kv_append): K against the 64-bit rotation,
V and every slot that no token goes to bit for bit."""
import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")

from decode_ref import assert_rounded, freqs, on_gpu, rotate  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _expected(k, v, kc, vc, table, pos, rows, rope):
    """CPU caches after the append (fp64 K with its bound) of [B, H, S, D] tokens; pos, rows [B, S]."""
    pages, H, ps, D = kc.shape
    k64, e64, v2 = kc.double(), torch.zeros_like(kc, dtype=torch.float64), vc.clone()
    kr, ke = k.double(), torch.zeros_like(k, dtype=torch.float64)
    if rope is not None:
        kr, ke = rotate(k, pos[:, None, :], *rope)
    written = torch.zeros(pages, ps, dtype=torch.bool)
    for b in range(k.shape[0]):
        for s in range(k.shape[2]):
            p, r = int(pos[b, s]), int(rows[b, s])
            if p < 0 or r < 0 or r >= table.shape[0] or p // ps >= table.shape[1]:
                continue
            page = int(table[r, p // ps])
            if page < 0 or page >= pages:
                continue
            k64[page, :, p % ps], e64[page, :, p % ps] = kr[b, :, s], ke[b, :, s]
            v2[page, :, p % ps] = v[b, :, s]
            written[page, p % ps] = True
    return k64, e64, v2, written


def _check(gpu_k, gpu_v, kc, expect):
    k64, e64, v2, written = expect
    got = gpu_k.cpu()
    assert torch.equal(gpu_v.cpu(), v2)
    keep = ~written[:, None, :, None].expand(got.shape)
    assert torch.equal(got[keep], kc[keep])
    assert_rounded(got, k64, e64)


CASES = [
    # B, H, S, D, page, rot, interleaved, order
    (5, 8, 1, 128, 16, 128, False, "phsd"),
    (3, 2, 70, 64, 24, 32, True, "pshd"),
    (2, 1, 33, 128, 1, 112, False, "phsd"),
    (1, 4, 257, 64, 7, 0, False, "pshd"),
    (4, 12, 9, 64, 256, 64, True, "phsd"),
    (70, 2, 1, 64, 5, 48, False, "pshd"),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_append_writes_its_slots_alone(case, dtype):
    B, H, S, D, ps, rot, inter, order = case
    print(f"[append] {case} {dtype}", flush=True)
    gen = torch.Generator().manual_seed(B * 100 + S)
    dt = TYPES[dtype]
    wide = -(-(S + 40) // ps)
    pages = B * wide + 3
    kc, vc = (torch.randn(pages, H, ps, D, generator=gen).to(dt) for _ in range(2))
    table = torch.randperm(pages, generator=gen)[:B * wide].view(B, wide).to(torch.int32)
    pos = torch.randint(0, 41, (B, 1), generator=gen) + torch.arange(S)
    pos[-1, S // 2:] = -1                  # padding
    pos[0, S - 1] = 2 ** 31 - 1 if B > 1 else pos[0, S - 1]  # beyond the table
    if wide > 1:
        table[B // 2, wide // 2] = -1      # no page
    if wide > 2:
        table[B // 2, 0] = pages           # no page either
        table[B // 2, 1] = -2 ** 31
    pos = pos.to(torch.int32)
    k, v = (torch.randn(B, S, H, D, generator=gen).to(dt).transpose(1, 2) for _ in range(2))
    rope = (freqs(rot), 1.1, inter) if rot else None
    kw = dict(inv_freq=rope[0].cuda(), rope_scale=1.1, interleaved=inter) if rot else {}
    rows = torch.arange(B)[:, None].expand(B, S)
    expect = _expected(k, v, kc, vc, table, pos, rows, rope)
    # token-major tensors, with a row for each batch entry
    gk, gv = on_gpu(kc, order), on_gpu(vc, order)
    seer.kv_append(k.cuda(), v.cuda(), gk, gv, table.cuda(), pos.cuda(), **kw)
    torch.cuda.synchronize()
    _check(gk, gv, kc, expect)
    # the same tokens packed, in another order, each with its row; head-major in memory
    perm = torch.randperm(B * S, generator=gen)
    pk, pv = (t.transpose(1, 2).reshape(B * S, H, D)[perm].transpose(0, 1).contiguous().transpose(0, 1).cuda()
              for t in (k, v))
    flat = lambda t: t.reshape(-1)[perm].to(torch.int32).cuda()
    gk, gv = on_gpu(kc, order), on_gpu(vc, order)
    seer.kv_append(pk, pv, gk, gv, table.cuda(), flat(pos), rows=flat(rows), **kw)
    torch.cuda.synchronize()
    _check(gk, gv, kc, expect)


def test_rows_outside_the_table_and_one_token_each():
    """Rows of -1 and beyond the table are padding; [B, H, D] tokens with [B] positions."""
    gen = torch.Generator().manual_seed(2)
    kc, vc = (torch.randn(9, 2, 8, 64, generator=gen) for _ in range(2))
    table = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32)
    k, v = (torch.randn(6, 2, 64, generator=gen) for _ in range(2))
    pos = torch.tensor([3, 15, 16, 0, 9, -3], dtype=torch.int32)
    rows = torch.tensor([2, 0, 1, -1, 3, 1], dtype=torch.int32)
    expect = _expected(k.unsqueeze(2), v.unsqueeze(2), kc, vc, table, pos[:, None], rows[:, None], None)
    gk, gv = kc.cuda(), vc.cuda()
    seer.kv_append(k.cuda(), v.cuda(), gk, gv, table.cuda(), pos.cuda(), rows=rows.cuda())
    _check(gk, gv, kc, expect)
    assert int(expect[3].sum()) == 2  # (row 2, position 3) and (row 0, position 15)
    # fewer tokens than table rows need no rows of their own
    gk, gv = kc.cuda(), vc.cuda()
    seer.kv_append(k[:2].cuda(), v[:2].cuda(), gk, gv, table.cuda(), pos[:2].cuda())
    _check(gk, gv, kc, _expected(k[:2].unsqueeze(2), v[:2].unsqueeze(2), kc, vc, table, pos[:2, None],
                                 torch.tensor([[0], [1]]), None))
    # and none at all is no call
    seer.kv_append(k[:0].cuda(), v[:0].cuda(), gk, gv, table.cuda(), pos[:0].cuda())


def test_cache_of_more_than_32_bits_of_elements():
    """Pages whose elements lie past 2^32 of each pool."""
    H, ps, D = 8, 128, 128
    pages = (1 << 32) // (H * ps * D) + 8
    print("[append] long cache", flush=True)
    kc, vc = (torch.empty(pages, H, ps, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kc[pages - 8:], vc[pages - 8:] = 0, 0
    gen = torch.Generator().manual_seed(4)
    k, v = (torch.randn(1, H, 3, D, generator=gen).bfloat16() for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device="cuda")
    pos = torch.tensor([[127, 128, 200]], dtype=torch.int32, device="cuda")
    seer.kv_append(k.cuda(), v.cuda(), kc, vc, table, pos)
    for new, pool in ((k, kc), (v, vc)):
        assert torch.equal(pool[pages - 1, :, 127].cpu(), new[0, :, 0])
        assert torch.equal(pool[pages - 3, :, 0].cpu(), new[0, :, 1])
        assert torch.equal(pool[pages - 3, :, 72].cpu(), new[0, :, 2])
        assert int(torch.count_nonzero(pool[pages - 8:])) == 3 * H * D - int((new == 0).sum())


def test_layouts_are_checked():
    k = torch.zeros(2, 2, 3, 64, device="cuda")
    kc = torch.zeros(4, 2, 8, 64, device="cuda")
    table, pos = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    ok = lambda **kw: seer.kv_append(*[kw.get(n, d) for n, d in (("k", k), ("v", k), ("kc", kc), ("vc", kc), ("table", table),
                                                                  ("pos", pos))], rows=kw.get("rows"))
    ok()
    for bad in (dict(kc=kc[:, :1]), dict(vc=kc[:2]), dict(kc=kc[0]), dict(pos=pos[:1]), dict(pos=pos[0]),
                dict(table=table[0]), dict(rows=pos[:1]), dict(table=table.cpu()), dict(kc=kc.cpu(), vc=kc.cpu()),
                dict(pos=torch.zeros(3, 2, dtype=torch.int32, device="cuda").t())):
        with pytest.raises(ValueError):
            ok(**bad)
    for bad in (dict(pos=pos.long()), dict(table=table.float()), dict(kc=kc.bfloat16(), vc=kc.bfloat16())):
        with pytest.raises(TypeError):
            ok(**bad)
    with pytest.raises(seer.SeerError) as e:
        ok(kc=kc[:1].expand(4, 2, 8, 64), vc=kc[:1].expand(4, 2, 8, 64))  # every page at one place
    assert e.value.status == seer.ERR_INVALID_ARG
    with pytest.raises(seer.SeerError) as e:
        ok(table=table[:1])
    assert e.value.status == seer.ERR_INVALID_ARG
