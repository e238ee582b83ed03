"""How far the calls over a cache in 4 bits are off in the mean (CPU, fp64): 2-norms over the elements of a call, where bounds for
single elements (cache_ref) have to add up all roundings as if they had one sign.

A rounding to fp32 is off by U = 2^-24 of the value at most, evenly spread within the last bit: U / sqrt(3) in the mean at a
mantissa of 1, half that at 2, 0.42 U over all mantissas (STEP).  A chain that sums n terms of either sign, of 2-norm T, holds T sqrt(i / n)
after i of them, so that its n roundings leave STEP sqrt(n / 2) T.  Errors of different sources add as squares.  What is
measured is allowed MARGIN times that.  (Where a source's count of roundings is not plain, the larger is taken: the stated arithmetic is
at a fifth to a half of what it is allowed, which test_cache_tight shows, with what the bounds do not let through.)"""
import math

import torch

import cache_ref as R
from decode_ref import U, rotate

STEP = 0.42 * U
MARGIN = 1.5


def terms(c, step, centred):
    """Sizes of what codes [.., D] add to a sum of products: in units of a step 16 + c, or 31 - c where a code enters
    complemented, 24 in the mean; centred codes within (c - 7.5) + 1 / 2."""
    size = (c.double() - 7.5).abs() + 0.5 if centred else torch.full(c.shape, 24.0, dtype=torch.float64)
    return size * step.repeat_interleave(c.shape[-1] // step.shape[-1], -1)


def score_error(c, step, mid, q, scale, centred, turned, parts):
    """Of scaled scores of a row q [D] (fp64, rotated) with keys [n, ..]: [n].  The products of each group's channels are summed,
    as many roundings as q has elements that are not 0, the groups' sums weighed with steps and added up (16 more); middles meet
    sums of q within a group.  The products of q's lesser parts (of `parts`) are added to what the sums start from, 24 steps (centred: 1 / 2)
    times the group's sum.  A rotated element is off by 2 U of its plane's length (cosine, sine, two products, a sum)."""
    ng = step.shape[-1]
    norms = (q ** 2).reshape(ng, -1).sum(-1)
    start2 = ((0.5 if centred else 24.0) ** 2 * step ** 2 * norms).sum(-1)
    value = R.stand_for(c, step, mid, c.shape[-1] // ng)
    t2 = ((q * terms(c, step, centred)) ** 2).sum(-1)
    a2 = (mid ** 2 * norms).sum(-1)
    x2 = (value @ q) ** 2
    n = int((q != 0).sum())
    e2 = STEP ** 2 * ((n / 2 + 8) * (t2 + x2 / 3) + (parts - 1) * n * start2 + 16 * (a2 + x2))
    if turned:
        e2 = e2 + (2 * U) ** 2 * ((q ** 2).sum() / max(int((q != 0).sum()), 1)) * (value ** 2 * (q != 0)).sum(-1)
    return scale * e2.sqrt()


def attend(q, kpool, vpool, table, page, pos, scale, turn=None, centred=None):
    """(o, lse, what o's elements and lse are off by in the mean, before o's rounding) of q [B, Hq, S, D] (CPU): fp64."""
    B, Hq, S, D = q.shape
    centred = q.dtype == torch.float32 if centred is None else centred
    parts = 1 if q.dtype == torch.bfloat16 and turn is None else 3
    (kc, ks, km), (vc, vs, vm) = R.opened(kpool), R.opened(vpool)
    k, v = R.values(kpool), R.values(vpool)
    pages, Hkv = k.shape[:2]
    scale = scale if scale > 0 else 1.0 / math.sqrt(D)
    o, eo = (torch.zeros(B, Hq, S, D, dtype=torch.float64) for _ in range(2))
    lse, el = torch.full((B, Hq, S), -math.inf, dtype=torch.float64), torch.zeros(B, Hq, S, dtype=torch.float64)
    for b in range(B):
        n = int(pos[b].max()) + 1
        if n <= 0:
            continue
        rows = [R.rows_of(x, table[b], page, n) for x in (kc, ks, km, vc, vs, vm, k, v)]
        for s in range(S):
            seen = R.seen_of(table[b], page, pages, int(pos[b, s]), n)
            for h in range(Hq):
                c, st, mi, cv, sv, mv, kk, vv = (x[seen, h // (Hq // Hkv)] for x in rows)
                qq = q[b, h, s].double()
                if turn is not None:
                    qq = rotate(q[b, h, s], pos[b, s], *turn)[0]
                x = scale * (kk @ qq)
                w = torch.softmax(x, 0)
                o[b, h, s], lse[b, h, s] = w @ vv, torch.logsumexp(x, 0)
                # a weight: its score, the argument of its power, the power
                d2 = score_error(c, st, mi, qq, scale, centred, turn is not None, parts) ** 2 + (STEP * (x - x.max())) ** 2 + U ** 2
                el[b, h, s] = ((w ** 2 * d2).sum() + (1.5 * U * lse[b, h, s]) ** 2 + U ** 2).sqrt()
                m = w.shape[0]
                tiles = -(-m // 64)
                t2 = (w[:, None] ** 2 * terms(cv, sv, centred) ** 2).sum(0)
                m2 = ((w[:, None] * mv) ** 2).sum(0).repeat_interleave(D // mv.shape[1])
                o2 = o[b, h, s] ** 2
                # sums of a tile's 64 products, of tiles, of wavefronts and workgroups (bf16: one sum over the tiles); of middles;
                # of the weights themselves
                e2 = (w[:, None] ** 2 * d2[:, None] * (vv - o[b, h, s]) ** 2).sum(0)
                sums = 32 + tiles / 2 if centred else m / 2
                e2 += STEP ** 2 * ((sums + 16) * (t2 + o2) + (m / 32 + 16) * (m2 + o2) + (tiles / 3 + 10) * o2)
                if q.dtype == torch.bfloat16:  # a weight times its step in two rounded parts
                    away = (cv.double() - 7.5) * sv.repeat_interleave(D // sv.shape[1], -1)
                    e2 += 2.0 ** -36 * (w[:, None] ** 2 * away ** 2).sum(0)
                eo[b, h, s] = e2.sqrt()
    return o, lse, eo, el


def norm(x):
    return float(x.double().norm())


def beyond_rounding(o, ref):
    """How far o is from ref beyond half a step of bf16 at ref (o in fp32: beyond nothing).  An o that is off by e before it is
    rounded is beyond by |e| at most."""
    d = (o.cpu().double() - ref).abs()
    if o.dtype == torch.float32:
        return d
    # (a ref that the error takes to the next power of two has that one's step)
    step = torch.pow(2.0, torch.floor(torch.log2((ref.abs() * (1 + 2.0 ** -16)).clamp_min(1e-300))) - 8)
    return (d - step).clamp_min(0.0)


def check(o, lse, want, what=""):
    """o (before its rounding) and lse of the call are within MARGIN of what attend expects."""
    ro, rl, eo, el = want
    some = rl > -math.inf
    off, off_l = norm(beyond_rounding(o, ro)), norm((lse.cpu().double() - rl)[some])
    print(f"{what} o {off / norm(ro):.2e} (allowed {MARGIN * norm(eo) / norm(ro):.2e}), lse {off_l / norm(rl[some]):.2e} "
          f"({MARGIN * norm(el) / norm(rl[some]):.2e})")
    assert off <= MARGIN * norm(eo) and off_l <= MARGIN * norm(el)


def weigh(q, kpool, table, page, pos, lse, scale, turn=None, centred=None):
    """(weights [B, Hkv, room], what they are off by in the mean) of q [B, Hq, S, D] over a Q4Pool: fp64.  A term's argument is
    rounded when the row's log-sum-exp is taken off and when it is scaled to base 2, whose factor is off by U / 4."""
    B, Hq, S, D = q.shape
    centred = q.dtype == torch.float32 if centred is None else centred
    parts = 1 if q.dtype == torch.bfloat16 and turn is None else 3
    kc, ks, km = R.opened(kpool)
    k = R.values(kpool)
    pages, Hkv = k.shape[:2]
    scale = scale if scale > 0 else 1.0 / math.sqrt(D)
    w = torch.zeros(B, Hkv, table.shape[1] * page, dtype=torch.float64)
    e2 = torch.zeros_like(w)
    for b in range(B):
        n = int(pos[b].max()) + 1
        if n <= 0:
            continue
        rows = [R.rows_of(x, table[b], page, n) for x in (kc, ks, km, k)]
        for s in range(S):
            seen = R.seen_of(table[b], page, pages, int(pos[b, s]), n)
            for h in range(Hq):
                g = h // (Hq // Hkv)
                c, st, mi, kk = (x[:, g] for x in rows)
                qq = q[b, h, s].double() if turn is None else rotate(q[b, h, s], pos[b, s], *turn)[0]
                x = scale * (kk @ qq) - float(lse[b, h, s])
                p = torch.where(seen, torch.exp(x), 0.0)
                d2 = score_error(c, st, mi, qq, scale, centred, turn is not None, parts) ** 2 + (U * x) ** 2 + U ** 2
                w[b, g, :n] += p
                e2[b, g, :n] += p ** 2 * d2
    return w, (e2 + (Hq // Hkv * S + 8) * (STEP * w) ** 2).sqrt()


def outlier_pool(seer, gen, pages, heads, page, dim, group, device="cuda"):
    """A Q4Pool whose groups hold one element of a code at the border, which the step was made for, and else elements near the
    middle, of codes 7 and 8: what a channel much larger than its neighbours leaves of them."""
    c = 7 + torch.randint(0, 2, (pages, heads, page, dim // group, group), generator=gen)
    at = torch.randint(0, group, c.shape[:-1], generator=gen)[..., None]
    c.scatter_(-1, at, 15 * torch.randint(0, 2, at.shape, generator=gen))
    c = c.reshape(pages, heads, page, dim).to(torch.uint8)
    params = torch.empty(pages, heads, page, dim // group, 2)
    params[..., 0] = 0.4 + 0.4 * torch.rand(params.shape[:-1], generator=gen)
    params[..., 1] = 0.1 * torch.randn(params.shape[:-1], generator=gen)
    return seer.Q4Pool((c[..., 0::2] | c[..., 1::2] << 4).to(device), params.to(torch.bfloat16).to(device))


def random_pool(seer, gen, pages, heads, page, dim, group, device="cuda"):
    p = torch.empty(pages, heads, page, dim // group, 2)
    p[..., 0] = 0.1 + 0.2 * torch.rand(p.shape[:-1], generator=gen)
    p[..., 1] = 0.3 * torch.randn(p.shape[:-1], generator=gen)
    return seer.Q4Pool(torch.randint(0, 256, (pages, heads, page, dim // 2), generator=gen, dtype=torch.uint8).to(device),
                       p.to(torch.bfloat16).to(device))
