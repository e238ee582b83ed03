"""Prefill and generation as a program runs them: pre-RoPE q and k to the gate, rope, sparse attention, the prompt's keys
and values into the cache, then token after token through kv_append and paged_attn, eager and as a replayed
graph, against dense attention in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")

from decode_ref import HALF_STEP, U, assert_rounded, freqs, rotate  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _dense(q, k, v):
    """fp64 attention of q [H, D] over k, v [n, Hkv, D] and sum p |v|."""
    g = q.shape[0] // k.shape[1]
    kk, vv = (t.repeat_interleave(g, 1).transpose(0, 1) for t in (k, v))
    p = torch.softmax((kk @ q.unsqueeze(-1)).squeeze(-1) / math.sqrt(q.shape[1]), -1).unsqueeze(1)
    return (p @ vv)[:, 0], (p @ vv.abs())[:, 0], (kk.abs() @ q.abs().unsqueeze(-1)).amax() / math.sqrt(q.shape[1])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_prompt_then_tokens(dtype):
    """Two prompts of unequal length and six tokens each.  Bound of o: keys and queries are rotated values rounded once
    (keys to the cache's type), so a score is off by (4 half steps of the cache's type + (D + 30) u) sum |q k| scale, a weight by
    twice that, and o by that times sum p |v|, beyond the sums of decode_ref."""
    dt = TYPES[dtype]
    B, Hq, Hkv, D, ps, steps = 2, 8, 2, 128, 16, 6
    lengths = [300, 77]
    print(f"[generation] {dtype}", flush=True)
    gen = torch.Generator().manual_seed(7)
    n = max(lengths)
    new = [torch.randn(B, h, n + steps, D, generator=gen).to(dt) for h in (Hq, Hkv, Hkv)]
    q, k, v = (t.cuda() for t in new)
    f = freqs(D, 500000.0)
    fg = f.cuda()
    wq = torch.randn(Hq, D, 64, generator=gen).cuda() / 8
    wk = torch.randn(Hkv, 3 * D, 64, generator=gen).cuda() / 8
    kc, vc = seer.alloc_kv_cache(2 * 24 + 2, ps, Hkv, D, dtype=dt)
    kc.fill_(float("nan")), vc.fill_(float("nan"))
    table = torch.randperm(50, generator=gen)[:48].view(2, 24).to(torch.int32).cuda()

    # the prompts, padded to the longer: gate on unrotated q and k, every block kept, then attention
    qp, kp, vp = (t[:, :, :n].contiguous() for t in (q, k, v))
    qr, kr = seer.rope(qp, kp, fg)
    mask = seer.gate(qp, kp, wq, wk, mode=seer.TOPK_RATIO, topk_ratio=1.0, rope_theta=500000.0)
    o, _ = seer.bsattn(qr, kr, vp, mask)
    pos = torch.arange(n, dtype=torch.int32).expand(B, n).clone()
    for b, m in enumerate(lengths):
        pos[b, m:] = -1
    seer.kv_append(kr, vp, kc, vc, table, pos.cuda())
    # the last prompt token by both attentions: the same sums in another order
    last = torch.tensor([[m - 1] for m in lengths], dtype=torch.int32).cuda()
    ql = torch.stack([qr[b, :, m - 1:m] for b, m in enumerate(lengths)])
    op, _ = seer.paged_attn(ql, kc, vc, table, last)
    for b, m in enumerate(lengths):
        # (prefill rounds P to bf16: a half step more of each)
        tol = 3 * HALF_STEP[dt] * float(vp[b].abs().max())
        assert float((op[b, :, 0].float() - o[b, :, m - 1].float()).abs().max()) <= tol

    # tokens: rotation on the way into the cache and in the attention
    r, _ = rotate(new[1], torch.arange(n + steps), f)
    rq, _ = rotate(new[0], torch.arange(n + steps), f)
    at = torch.tensor(lengths, dtype=torch.int32).cuda()  # the next token's position, advanced on the device
    for t in range(steps):
        src = [m + t for m in lengths]
        q1, k1, v1 = (torch.stack([x[b, :, p] for b, p in enumerate(src)]) for x in (q, k, v))
        seer.kv_append(k1, v1, kc, vc, table, at, inv_freq=fg)
        o1, _ = seer.paged_attn(q1, kc, vc, table, at, inv_freq=fg)
        at += 1
        for b, p in enumerate(src):
            ref, size, a = _dense(rq[b, :, p], r[b, :, :p + 1].transpose(0, 1), new[2][b, :, :p + 1].double().transpose(0, 1))
            err = (2 * (4 * HALF_STEP[dt] + (D + 30) * U) * a + 2 * (p + 9) * U + 2.0 ** -16) * size
            assert_rounded(o1[b].cpu(), ref, err, f"token {t} of sequence {b}")


def test_captured_step_replays_with_new_positions():
    """append + attention captured once; every replay, with eager work and a synchronisation in between, equals the eager
    calls on the same state bit for bit, while the sequences grow across page ends."""
    B, Hq, Hkv, D, ps = 3, 8, 2, 128, 16
    gen = torch.Generator(device="cuda").manual_seed(3)
    fg = freqs(D).cuda()
    kc, vc = (torch.randn(3 * 100, Hkv, ps, D, device="cuda", generator=gen).bfloat16() for _ in range(2))
    table = torch.randperm(300, device="cuda", generator=gen).view(3, 100).to(torch.int32)
    at = torch.tensor([13, 1500, 700], dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros(B, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    out, lse = torch.empty_like(q), torch.empty(B, Hq, device="cuda")
    qo, ko = torch.empty_like(q).unsqueeze(2), torch.empty_like(k).unsqueeze(2)

    def step():
        seer.rope(q.unsqueeze(2), k.unsqueeze(2), fg, at[:, None], out=(qo, ko))
        seer.kv_append(ko, v.unsqueeze(2), kc, vc, table, at)
        seer.paged_attn(qo[:, :, 0], kc, vc, table, at, out=out, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for r in range(5):
        print(f"[generation] replay {r}", flush=True)
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
        saved = kc.clone(), vc.clone()
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, kc, vc)]
        kc.copy_(saved[0]), vc.copy_(saved[1])
        out.zero_(), lse.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, lse, kc, vc)):
            assert torch.equal(a, b)
        at += 1


def test_given_and_side_streams():
    """Calls on a given stream and under a side stream equal those on the default one, memory of their own included."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    fg = freqs(64).cuda()
    kc, vc = (torch.randn(80, 2, 16, 64, device="cuda", generator=gen) for _ in range(2))
    table = torch.arange(80, device="cuda", dtype=torch.int32).view(1, 80)
    q = torch.randn(1, 4, 2, 64, device="cuda", generator=gen)
    k = torch.randn(1, 2, 2, 64, device="cuda", generator=gen)
    pos = torch.tensor([[1200, 1201]], dtype=torch.int32, device="cuda")

    def work(stream=None):
        a, b = seer.rope(q, k, fg, pos, stream=stream)
        seer.kv_append(b, k, kc, vc, table, pos, stream=stream)
        return [a, b, *seer.paged_attn(a, kc, vc, table, pos, want_lse=True, stream=stream)]

    want = work()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = work(s)
    s.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        under = work()
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, under):
        assert torch.equal(a, b) and torch.equal(a, c)
