"""Plain 64-bit forms of the cache in 4 bits, attention over it, the weights of cached keys and eviction (CPU tensors), and how
far an implementation in the stated arithmetic can be from them.

U = 2^-24 is half a step of fp32 relative to the value; bf16's is 2^-8."""
import math

import torch

from decode_ref import U, rotate


def quantise(x, group):
    """(codes, step, middle) of x [.., D] (bf16 or fp32) by the definition: step and middle [.., D / group] (fp64)."""
    y = x.double().reshape(*x.shape[:-1], -1, group)
    hi, lo = y.amax(-1), y.amin(-1)
    fine = (y.abs() <= 2.0 ** 127).all(-1)
    hi, lo = torch.where(fine, hi, 0.0), torch.where(fine, lo, 0.0)
    y = torch.where(fine[..., None], y, 0.0)
    mid = (hi.float() * 0.5 + lo.float() * 0.5).to(torch.bfloat16).double()
    reach = torch.maximum(hi - mid, mid - lo)
    # the least number of 8 significant bits that is reach / 7.5 or more: 7.5 times it is exact, so the comparison is
    s = reach / 7.5
    e = torch.floor(torch.log2(s.clamp_min(1e-300)))
    step = torch.full_like(s, math.inf)
    for de in (-1, 0, 1):
        unit = torch.pow(torch.tensor(2.0, dtype=torch.float64), e + de - 7)
        for up in (-1, 0, 1, 2):
            c = (torch.floor(s / unit) + up) * unit
            whole = c / unit <= 256
            step = torch.where((c * 7.5 >= reach) & whole & (c < step), c, step)
    step = torch.where(reach > 0, step.clamp_min(2.0 ** -100), 0.0)
    d = y - mid[..., None]
    c = torch.zeros(y.shape, dtype=torch.int64)
    for b in range(-7, 8):
        c += (d >= b * step[..., None]).long()
    c = torch.where(step[..., None] > 0, c, 8)
    step = torch.where(fine, step, math.nan)
    mid = torch.where(fine, mid, 0.0)
    c = torch.where(fine[..., None], c, 8)
    return c.reshape(x.shape), step, mid


def stand_for(codes, step, mid, group):
    """The values that codes [.., D] stand for (fp64)."""
    c = codes.double().reshape(*codes.shape[:-1], -1, group)
    return (mid[..., None] + step[..., None] * (c - 7.5)).reshape(codes.shape)


def opened(pool):
    """(codes [.., D], step, middle [.., D / group]) (int64, fp64) of a Q4Pool, on the CPU."""
    c = pool.codes.cpu().long()
    c = torch.stack((c & 15, c >> 4), -1).flatten(-2)
    p = pool.params.cpu().double()
    return c, p[..., 0], p[..., 1]


def values(pool):
    """What a pool (Q4Pool or tensor) stands for: fp64 [pages, heads, slots, D], on the CPU."""
    if hasattr(pool, "codes"):
        c, s, m = opened(pool)
        return stand_for(c, s, m, c.shape[-1] // s.shape[-1])
    return pool.cpu().double()


def size(pool):
    """What an element of a pool weighs in the sums that its products run through (fp64, like values): in 4 bits a code enters as
    1 + c / 16 < 2 of 16 steps, 32 steps, and the middle and what takes the 1 out again, 1.5 of 16 steps, beside it."""
    if not hasattr(pool, "codes"):
        return pool.cpu().double().abs()
    c, s, m = opened(pool)
    g = c.shape[-1] // s.shape[-1]
    return (56 * s + m.abs()).repeat_interleave(g, -1)


def random_pool(seer, gen, pages, heads, page, dim, group, order="phsd"):
    """A Q4Pool (on the GPU) of random codes."""
    codes = torch.randint(0, 256, (pages, heads, page, dim // 2), generator=gen, dtype=torch.uint8)
    params = torch.empty(pages, heads, page, dim // group, 2)
    params[..., 0] = 0.1 + 0.2 * torch.rand(params.shape[:-1], generator=gen)
    params[..., 1] = 0.3 * torch.randn(params.shape[:-1], generator=gen)
    params = params.to(torch.bfloat16)
    if order == "pshd":
        codes = codes.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        params = params.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        return seer.Q4Pool(codes, params)
    return seer.Q4Pool(codes.cuda(), params.cuda())


def paged(gen, lengths, page, spare=2, wide=None):
    """(table int32 [B, wide], pages of the pool, pages that none holds) for sequences of these lengths, in no order."""
    used = [-(-n // page) if n > 0 else 0 for n in lengths]
    pages = sum(used) + spare
    wide = wide or max(max(used), 1)
    perm = torch.randperm(pages, generator=gen).tolist()
    table = torch.full((len(lengths), wide), -1, dtype=torch.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = torch.tensor(perm[at:at + u], dtype=torch.int32)
        at += u
    return table, pages, perm[at:]


def seen_of(table, page, pages, pos, n):
    """Which of a sequence's first n slots a token at pos sees."""
    t = torch.arange(n)
    p = table[torch.div(t, page, rounding_mode="floor")].long()
    return (p >= 0) & (p < pages) & (t <= pos)


def rows_of(x, table, page, n):
    """[n, heads, ..] of a sequence's first n slots of x [pages, heads, slots, ..] (slots of no page: any)."""
    t = torch.arange(n)
    p = table[torch.div(t, page, rounding_mode="floor")].long().clamp(0, x.shape[0] - 1)
    return x[p, :, t % page]


def score(q, k, ks, scale, turn, dtype, pos):
    """Scaled scores of a row q [D] with keys k [n, D] and a bound on their error.  A score is a sum of D terms (and as many
    for the groups), in fp32, each rounded: (2 D + 16) U of scale sum |q| size(k); its scaling and the argument of the power 4 U
    (1 + |s|).  turn: (freqs, scale, interleaved): q is rotated first, off by rotate's bound, and enters whole."""
    qq, eq = q.double(), torch.zeros(q.shape, dtype=torch.float64)
    if turn is not None:
        qq, eq = rotate(q, pos, *turn)
        eq = eq + U * qq.abs()
    x = scale * (k @ qq)
    d = (2 * q.shape[-1] + 16) * U * scale * (ks @ qq.abs()) + 4 * U * (1 + x.abs()) + scale * (ks @ eq)
    return x, d


def attend(q, kpool, vpool, table, page, pos, scale, turn=None, rope_pos=None):
    """fp64 attention of q [B, Hq, S, D] (CPU) over pools in 4 bits: o, lse and their bounds.

    A weight is off by twice its score's error relative to the maximum's and 4 U of the power; o's sums of n terms by (2 n + 16)
    U of sum p size(v) / sum p; a weight times its step enters whole (fp32) or in two rounded bf16 parts, 2^-18 of it off."""
    B, Hq, S, D = q.shape
    k, v, ks, vs = values(kpool), values(vpool), size(kpool), size(vpool)
    pages, Hkv = k.shape[:2]
    cap = table.shape[1] * page
    scale = scale if scale > 0 else 1.0 / math.sqrt(D)
    o = torch.zeros(B, Hq, S, D, dtype=torch.float64)
    eo = torch.zeros_like(o)
    lse = torch.full((B, Hq, S), -math.inf, dtype=torch.float64)
    el = torch.zeros_like(lse)
    rope_pos = pos if rope_pos is None else rope_pos
    for b in range(B):
        n = min(int(pos[b].max()) + 1, cap)
        if n <= 0:
            continue
        kb, vb, ksb, vsb = (rows_of(x, table[b], page, n) for x in (k, v, ks, vs))
        for s in range(S):
            seen = seen_of(table[b], page, pages, int(pos[b, s]), n)
            if not bool(seen.any()):
                continue
            for h in range(Hq):
                g = h // (Hq // Hkv)
                x, d = score(q[b, h, s], kb[seen, g], ksb[seen, g], scale, turn, q.dtype, rope_pos[b, s])
                m = x.shape[0]
                p = torch.exp(x - x.max())
                L = p.sum()
                dd = float(d.max())
                o[b, h, s] = p @ vb[seen, g] / L
                lse[b, h, s] = x.max() + torch.log(L)
                el[b, h, s] = dd + (m + 8) * U * (1 + abs(float(lse[b, h, s])))
                part = 2.0 ** -18 if q.dtype == torch.bfloat16 else 0.0
                eo[b, h, s] = (2 * dd + (2 * m + 24) * U + part) * (p @ vsb[seen, g] / L)
    return o, lse, eo, el


def weigh(q, kpool, table, page, pos, lse, before, decay, scale, width, turn=None, rope_pos=None):
    """fp64 weights [B, Hkv, W] after kv_weights, and their bound (entries that stay: bound 0)."""
    B, Hq, S, D = q.shape
    k, ks = values(kpool), size(kpool)
    pages, Hkv = k.shape[:2]
    cap = min(table.shape[1] * page, width)
    scale = scale if scale > 0 else 1.0 / math.sqrt(D)
    w = before.double().clone()
    e = torch.zeros_like(w)
    rope_pos = pos if rope_pos is None else rope_pos
    for b in range(B):
        n = min(int(pos[b].max()) + 1, cap)
        if n <= 0:
            continue
        kb, ksb = rows_of(k, table[b], page, n), rows_of(ks, table[b], page, n)
        for g in range(Hkv):
            total, err = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
            rows = 0
            for s in range(S):
                seen = seen_of(table[b], page, pages, int(pos[b, s]), n)
                for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                    if float(lse[b, h, s]) == -math.inf:
                        continue
                    x, d = score(q[b, h, s], kb[:, g], ksb[:, g], scale, turn, q.dtype, rope_pos[b, s])
                    p = torch.where(seen, torch.exp(x - float(lse[b, h, s])), 0.0)
                    total += p
                    # the row's log-sum-exp is scaled and subtracted in fp32; the power adds 4 U
                    err += torch.where(seen, p * (d + U * (4 * abs(float(lse[b, h, s])) + 4 * x.abs() + 8)) * 1.01, 0.0)
                    rows += 1
            old = decay * before[b, g, :n].double() if decay else torch.zeros(n, dtype=torch.float64)
            w[b, g, :n] = old + total
            e[b, g, :n] = err + (rows + 8) * U * total + 2 * U * (old.abs() + total)
    return w, e


def evict(weights, lengths, keep, first, last, cap):
    """kept slots (lists by sequence and head)."""
    out = []
    for b, n in enumerate(lengths):
        n = min(max(n, 0), cap)
        heads = []
        for h in range(weights.shape[1]):
            w = [float(weights[b, h, i]) if i < weights.shape[2] else 0.0 for i in range(n)]
            if n <= keep:
                heads.append(list(range(n)))
                continue
            free = range(first, n - last)
            rank = sorted(free, key=lambda i: (-math.inf if math.isnan(w[i]) else -w[i], 0 if math.isnan(w[i]) else 1, i))
            heads.append(sorted(list(range(first)) + rank[:keep - first - last] + list(range(n - last, n))))
        out.append(heads)
    return out
