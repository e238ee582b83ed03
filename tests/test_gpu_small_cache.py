"""The calls that keep a cache small as they are used together, in graphs, on streams, and over layouts that the other tests do
not have."""
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


def close_lse(lse, ref, bound):
    d = (lse.cpu().double() - ref).abs()
    assert bool((d <= bound + R.U * ref.abs()).all())


@pytest.mark.parametrize("kind", ["q4", "bf16"])
def test_a_prompt_its_eviction_and_the_answer(kind):
    """A prompt goes into the cache, its last tokens weigh the keys, the cache is cut, and new tokens are stored at slots that
    are not their positions, attended over and weighed: every call against the 64-bit forms of what the cache then holds."""
    gen = torch.Generator().manual_seed(1)
    B, Hq, Hkv, D, page, keep, first, last = 2, 4, 2, 128, 16, 40, 2, 8
    lengths = [100, 61]
    f = freqs(D, 500000.0)
    dt = torch.bfloat16
    n32 = torch.tensor(lengths, dtype=torch.int32).cuda()
    room = 7 + 4  # pages of a sequence before and after
    table = torch.arange(B * 7, dtype=torch.int32).reshape(B, 7)
    new = (B * 7 + torch.arange(B * 4, dtype=torch.int32)).reshape(B, 4)
    if kind == "q4":
        kc, vc = (R.random_pool(seer, gen, B * room, Hkv, page, D, 32) for _ in range(2))
    else:
        kc, vc = (torch.randn(B * room, Hkv, page, D, generator=gen).to(dt).cuda() for _ in range(2))
    k, v = (torch.randn(B, Hkv, 100, D, generator=gen).to(dt).cuda() for _ in range(2))
    pos = torch.stack([torch.where(torch.arange(100) < n, torch.arange(100), -1) for n in lengths]).to(torch.int32)
    kr = seer.rope(k, None, f.cuda(), positions=pos.cuda())[0]
    store = seer.kv_append_q4 if kind == "q4" else seer.kv_append
    store(kr, v, kc, vc, table.cuda(), pos.cuda())
    # the prompt's last 5 tokens weigh all keys
    q = torch.randn(B, Hq, 5, D, generator=gen).to(dt)
    at = (torch.tensor(lengths)[:, None] - 5 + torch.arange(5)).to(torch.int32)
    attn = seer.paged_attn_q4 if kind == "q4" else seer.paged_attn
    _, lse = attn(q.cuda(), kc, vc, table.cuda(), at.cuda(), want_lse=True)
    w = torch.zeros(B, Hkv, 7 * page).cuda()
    seer.kv_weights(q.cuda(), kc, table.cuda(), at.cuda(), lse, w, decay=0.0)
    ref, err = R.weigh(q, kc, table, page, at, lse.cpu(), torch.zeros(B, Hkv, 7 * page), 0.0, 0.0, 7 * page)
    assert bool(((w.cpu().double() - ref).abs() <= err).all())
    # the cut
    old = [R.values(kc), R.values(vc)]
    new_n, kept, w2 = seer.kv_evict(kc, vc, table.cuda(), n32, w, new.cuda(), keep, first=first, last=last)
    want = R.evict(w.cpu(), lengths, keep, first, last, 7 * page)
    assert new_n.tolist() == [keep, keep]
    for b in range(B):
        for h in range(Hkv):
            assert kept[b, h].tolist() == want[b][h]
            for x, y in zip(old, (R.values(kc), R.values(vc))):
                assert torch.equal(R.rows_of(y, new[b], page, keep)[:, h], R.rows_of(x, table[b], page, 100)[want[b][h], h])
    # three more tokens, at positions 100 .. and 61 .., slots 40 ..
    for step in range(3):
        slots = torch.full((B,), keep + step, dtype=torch.int32)
        places = torch.tensor(lengths, dtype=torch.int32) + step
        k1, v1 = (torch.randn(B, Hkv, D, generator=gen).to(dt).cuda() for _ in range(2))
        q1 = torch.randn(B, Hq, D, generator=gen).to(dt)
        if kind == "q4":
            seer.kv_append_q4(k1, v1, kc, vc, new.cuda(), slots.cuda(), inv_freq=f.cuda(), rope_positions=places.cuda())
            o, lse = seer.paged_attn_q4(q1.cuda(), kc, vc, new.cuda(), slots.cuda(), inv_freq=f.cuda(), rope_positions=places.cuda(),
                                        want_lse=True)
            ro, rl, eo, el = R.attend(q1[:, :, None], kc, vc, new, page, slots[:, None], 0.0, (f, 1.0, False), places[:, None])
            assert_rounded(o, ro[:, :, 0], eo[:, :, 0], "o")
            close_lse(lse, rl[:, :, 0], el[:, :, 0])
        else:
            q1t, k1t = seer.rope(q1.cuda()[:, :, None], k1[:, :, None], f.cuda(), positions=places.cuda()[:, None])
            seer.kv_append(k1t, v1[:, :, None], kc, vc, new.cuda(), slots.cuda()[:, None])
            o, lse = seer.paged_attn(q1t[:, :, 0], kc, vc, new.cuda(), slots.cuda(), want_lse=True)
            q1 = q1t[:, :, 0].cpu()
        turn = dict(inv_freq=f.cuda(), rope_positions=places.cuda()) if kind == "q4" else {}
        before = w2.cpu().clone()
        seer.kv_weights(q1.cuda(), kc, new.cuda(), slots.cuda(), lse, w2, **turn)
        ref, err = R.weigh(q1[:, :, None], kc, new, page, slots[:, None], lse.cpu()[:, :, None], before, 1.0, 0.0, 4 * page,
                           (f, 1.0, False) if kind == "q4" else None, places[:, None])
        assert bool(((w2.cpu().double() - ref).abs() <= err).all())


@pytest.mark.parametrize("room", [640, 40000])
def test_a_captured_step(room):
    """A step of generation and an eviction in a graph, replayed with new tokens, positions and lengths, with eager work in
    between: every replay is the eager result, bit for bit."""
    gen = torch.Generator().manual_seed(2)
    B, Hq, Hkv, D, page = 3, 8, 2, 64, 16
    table, pages, free = R.paged(gen, [room] * 3, page, spare=12)
    table, to = table.cuda(), torch.tensor(free[:12], dtype=torch.int32).reshape(3, 4).cuda()
    f = freqs(D).cuda()

    def state():
        g = torch.Generator().manual_seed(3)
        kc, vc = (R.random_pool(seer, g, pages, Hkv, page, D, 32) for _ in range(2))
        return kc, vc, torch.rand(B, Hkv, room, generator=g).cuda()

    def step(kc, vc, w, k1, v1, q1, slots, n):
        seer.kv_append_q4(k1, v1, kc, vc, table, slots, inv_freq=f)
        o, lse = seer.paged_attn_q4(q1, kc, vc, table, slots, inv_freq=f, want_lse=True)
        seer.kv_weights(q1, kc, table, slots, lse, w, inv_freq=f, decay=0.9)
        k, v = seer.kv_read(kc, vc, table, slots)
        return (o, lse, k, v, *seer.kv_evict(kc, vc, table, n, w, to, 60, first=1, last=3))

    def draw(i):
        g = torch.Generator().manual_seed(100 + i)
        x = [torch.randn(B, h, D, generator=g).to(torch.bfloat16).cuda() for h in (Hkv, Hkv, Hq)]
        slots = torch.randint(0, room, (B,), generator=g).to(torch.int32).cuda()
        return (*x, slots, torch.randint(0, room + 1, (B,), generator=g).to(torch.int32).cuda())

    mine, other = state(), state()
    args = draw(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*state(), *draw(9))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*mine, *args)
    for i in range(4):
        for a, x in zip(args, draw(i)):
            a.copy_(x)
        graph.replay()
        want = step(*other, *draw(i))
        torch.cuda.synchronize()
        for a, x in zip(out, want):
            assert torch.equal(a, x)
        for a, x in zip(mine, other):
            for s, t in ((a.codes, x.codes), (a.params.view(torch.int16), x.params.view(torch.int16))) if hasattr(a, "codes") else ((a, x),):
                assert torch.equal(s, t)


def test_two_streams():
    """Calls on two streams at once, each with tensors of its own, and the stream argument."""
    gen = torch.Generator().manual_seed(4)
    table, pages, _ = R.paged(gen, [3000, 900], 16)
    table = table.cuda()
    kc, vc = (R.random_pool(seer, gen, pages, 2, 16, 128, 32) for _ in range(2))
    pos = torch.tensor([2999, 899], dtype=torch.int32).cuda()
    qs = [torch.randn(2, 8, 128, generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
    want = [seer.paged_attn_q4(q, kc, vc, table, pos, want_lse=True) for q in qs]
    ww = [seer.kv_weights(q, kc, table, pos, x[1], torch.zeros(2, 2, 3008).cuda(), decay=0.0) for q, x in zip(qs, want)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got, gw = [[], []], [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            o, lse = seer.paged_attn_q4(qs[i], kc, vc, table, pos, want_lse=True, stream=s)
            got[i].append((o, lse))
            with torch.cuda.stream(s):
                gw[i].append(seer.kv_weights(qs[i], kc, table, pos, lse, torch.zeros(2, 2, 3008, device="cuda"), decay=0.0))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lse in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])
        for w in gw[i]:
            assert torch.equal(w, ww[i])


def far_pool(seer, gen, pages, page, dim, group):
    """A Q4Pool of one head whose pages are 2.5 GB apart (codes) and 1.25 GB (params)."""
    codes = torch.empty((pages - 1) * (5 << 29) + page * dim // 2, dtype=torch.uint8, device="cuda")
    params = torch.empty((pages - 1) * (5 << 28) + page * (dim // group) * 2, dtype=torch.bfloat16, device="cuda")
    ng = dim // group
    pool = seer.Q4Pool(codes.as_strided((pages, 1, page, dim // 2), (5 << 29, page * dim // 2, dim // 2, 1)),
                       params.as_strided((pages, 1, page, ng, 2), (5 << 28, page * ng * 2, ng * 2, 2, 1)))
    near = R.random_pool(seer, gen, pages, 1, page, dim, group)
    pool.codes.copy_(near.codes)
    pool.params.copy_(near.params)
    return pool, near


@pytest.mark.parametrize("page", [16, 12])
def test_pools_beyond_32_bits(page):
    """Pages whose offsets pass 32 bits: all calls give what they give on a small pool."""
    gen = torch.Generator().manual_seed(page)
    (kc, kn), (vc, vn) = (far_pool(seer, gen, 4, page, 128, 32) for _ in range(2))
    table = torch.tensor([[2, 3, 0]], dtype=torch.int32).cuda()
    to = torch.tensor([[1]], dtype=torch.int32).cuda()
    n = 3 * page - 2
    pos = torch.tensor([n - 1], dtype=torch.int32).cuda()
    q, k1, v1 = (torch.randn(1, h, 128, generator=gen).to(torch.bfloat16).cuda() for h in (4, 1, 1))
    out = []
    for a, b in ((kc, vc), (kn, vn)):
        seer.kv_append_q4(k1, v1, a, b, table, pos)
        o, lse = seer.paged_attn_q4(q, a, b, table, pos, want_lse=True)
        w = seer.kv_weights(q, a, table, pos, lse, torch.zeros(1, 1, 3 * page).cuda(), decay=0.0)
        read = seer.kv_read(a, b, table, torch.arange(n, dtype=torch.int32).cuda()[None])
        cut = seer.kv_evict(a, b, table, pos + 1, w, to, page - 3, last=2)
        out.append((o, lse, w, *read, *cut, a.codes, b.codes, a.params.view(torch.int16), b.params.view(torch.int16)))
    for x, y in zip(*out):
        assert torch.equal(x, y)


def test_broadcast_and_strided_operands():
    """Expanded heads and batches, rows of a wider tensor, outputs in another layout."""
    gen = torch.Generator().manual_seed(6)
    table, pages, _ = R.paged(gen, [40, 40], 8)
    kc, vc = (R.random_pool(seer, gen, pages, 4, 8, 64, 64) for _ in range(2))
    kd, vd = (seer.Q4Pool(p.codes.clone(), p.params.clone()) for p in (kc, vc))
    wide = torch.randn(2, 40, 200, generator=gen).to(torch.bfloat16).cuda()
    k = wide[:, None, :, 64:128].expand(2, 4, 40, 64)       # one head for all
    v = wide[:1, :, :192].reshape(1, 40, 3, 64).transpose(1, 2)[:, :1].expand(2, 4, 40, 64)
    pos = torch.arange(40, dtype=torch.int32).cuda().expand(2, 40)
    seer.kv_append_q4(k, v, kc, vc, table.cuda(), pos)
    seer.kv_append_q4(k.contiguous(), v.contiguous(), kd, vd, table.cuda(), pos.contiguous())
    assert torch.equal(kc.codes, kd.codes) and torch.equal(vc.codes, vd.codes)
    at = torch.full((1,), 39, dtype=torch.int32).cuda().expand(2)
    q = torch.randn(1, 1, 64, generator=gen).cuda().expand(2, 8, 64)
    o, lse = seer.paged_attn_q4(q, kc, vc, table.cuda(), at, want_lse=True, out=torch.empty(8, 2, 64).cuda().transpose(0, 1))
    o2, lse2 = seer.paged_attn_q4(q.contiguous(), kc, vc, table.cuda(), at.contiguous(), want_lse=True)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_the_call_refuses():
    """What the binding can see of tensors on the GPU."""
    kc, vc = seer.alloc_kv_cache_q4(4, 16, 2, 64)
    pk = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16).cuda()
    table = torch.zeros(2, 2, dtype=torch.int32).cuda()
    pos = torch.zeros(2, dtype=torch.int32).cuda()
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16).cuda()
    lse, w = torch.zeros(2, 2).cuda(), torch.zeros(2, 2, 32).cuda()
    to = torch.ones(2, 1, dtype=torch.int32).cuda()
    f = freqs(64)
    for error, call in (
            (TypeError, lambda: seer.kv_append_q4(k, k, pk, pk, table, pos)),                    # a cache of values
            (TypeError, lambda: seer.paged_attn_q4(k, pk, pk, table, pos)),
            (TypeError, lambda: seer.kv_append_q4(k.half(), k.half(), kc, vc, table, pos)),
            (ValueError, lambda: seer.kv_append_q4(k, k[:, :1], kc, vc, table, pos)),
            (ValueError, lambda: seer.kv_append_q4(k[:, :1], k[:, :1], kc, vc, table, pos)),       # heads
            (ValueError, lambda: seer.kv_append_q4(k, k, kc, seer.alloc_kv_cache_q4(4, 8, 2, 64)[0], table, pos)),
            (ValueError, lambda: seer.kv_append_q4(k, k, kc, seer.alloc_kv_cache_q4(4, 16, 2, 64, group=64)[0], table, pos)),
            (ValueError, lambda: seer.kv_append_q4(k, k, kc, pk, table, pos)),
            (TypeError, lambda: seer.kv_append_q4(k, k, kc, vc, table, pos.long())),
            (TypeError, lambda: seer.kv_append_q4(k, k, kc, vc, table.long(), pos)),
            (ValueError, lambda: seer.kv_append_q4(k, k, kc, vc, table, pos[:1])),
            (ValueError, lambda: seer.kv_append_q4(k, k, kc, vc, table, pos, rows=pos[:1])),
            (ValueError, lambda: seer.kv_append_q4(k, k, kc, vc, table, pos, rope_positions=pos.cpu()[:1])),
            (ValueError, lambda: seer.kv_append_q4(k, k, kc, vc, table, pos, inv_freq=f)),          # on the CPU
            (TypeError, lambda: seer.kv_read(pk, pk, table, pos, dtype=torch.float32)),
            (ValueError, lambda: seer.kv_read(kc, vc, table, pos[None, None])),
            (ValueError, lambda: seer.kv_read(kc, vc, table, pos, out=(k, k[:1]))),
            (TypeError, lambda: seer.kv_read(kc, vc, table, pos, dtype=torch.float16)),
            (ValueError, lambda: seer.paged_attn_q4(k, kc, vc, table[:1], pos)),
            (ValueError, lambda: seer.paged_attn_q4(k, kc, vc, table, pos, out=k[:1])),
            (ValueError, lambda: seer.paged_attn_q4(k, kc, vc, table, pos, lse=lse[:1])),
            (seer.SeerError, lambda: seer.paged_attn_q4(k, kc, vc, table, pos, workspace=torch.empty(1).cuda())),
            (seer.SeerError, lambda: seer.paged_attn_q4(k, kc, vc, table, pos, sm_scale=math.inf)),
            (TypeError, lambda: seer.kv_weights(k, kc, table, pos, lse, w.double())),
            (ValueError, lambda: seer.kv_weights(k, kc, table, pos, lse, w[:, :1])),
            (ValueError, lambda: seer.kv_weights(k, kc, table, pos, lse[:1], w)),
            (ValueError, lambda: seer.kv_weights(k, kc, table, pos, lse, w, out=w[..., :5])),
            (TypeError, lambda: seer.kv_weights(k.float(), pk, table, pos, lse, w)),                 # q in another type than values
            (ValueError, lambda: seer.kv_evict(kc, vc, table, pos, w, to, 17)),                      # no room
            (ValueError, lambda: seer.kv_evict(kc, vc, table, pos, w, to, 0)),
            (ValueError, lambda: seer.kv_evict(kc, vc, table, pos, w, to, 4, first=3, last=2)),
            (ValueError, lambda: seer.kv_evict(kc, vc, table, pos, w[:1], to, 4)),
            (ValueError, lambda: seer.kv_evict(kc, vc, table[:1], pos, w, to, 4)),
            (seer.SeerError, lambda: seer.kv_evict(kc, vc, table, pos, w, to, 4, out=(pos, torch.empty(2, 2, 4, dtype=torch.int32).cuda(), w)))):
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()
