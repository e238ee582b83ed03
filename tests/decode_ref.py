"""Plain 64-bit (angles: 80-bit) forms of the rotary positions, the paged append and paged
attention, and how far an implementation in the stated arithmetic can be from them.

u = 2^-24 is half a step of fp32 relative to the value; bf16's is 2^-8."""
import math

import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def freqs(rot, theta=10000.0):
    return torch.tensor([theta ** (-2.0 * p / rot) for p in range(rot // 2)], dtype=torch.float64)


def rotate(x, pos, f, scale=1.0, interleaved=False, grad=False):
    """x [.., D] (CPU) rotated at pos, which broadcasts over x's leading axes; returns (result, error bound), fp64.

    Bound: the cosine and sine of the reduced angle are within 3 u (series 2.5e-8, the angle's conversion and its product with
    2 pi 2^-32 u pi/4 each, the evaluation u), the scale's product, each product and the sum round once: 6 u (|x| + |y|) scale.
    The rate of a turn per position is held to 2^-53 twice over (1 / 2 pi and the product): pos f 2^-52 of angle."""
    rot = 2 * f.numel()
    ang = pos.numpy().astype(np.longdouble)[..., None] * f.numpy().astype(np.longdouble)
    c = torch.from_numpy(np.cos(ang).astype(np.float64))
    s = torch.from_numpy(np.sin(ang).astype(np.float64)) * (-1.0 if grad else 1.0)
    y = x.double()
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    a2, b2 = scale * (a * c - b * s), scale * (a * s + b * c)
    e = abs(scale) * (a.abs() + b.abs()) * (6 * U + torch.from_numpy(np.abs(ang).astype(np.float64)) * 2.0 ** -52)
    out, err = y.clone(), torch.zeros_like(y)
    if interleaved:
        out[..., 0:rot:2], out[..., 1:rot:2] = a2, b2
        err[..., 0:rot:2], err[..., 1:rot:2] = e, e
    else:
        out[..., :rot // 2], out[..., rot // 2:rot] = a2, b2
        err[..., :rot // 2], err[..., rot // 2:rot] = e, e
    return out, err


def assert_rounded(got, ref, err, what=""):
    """got is ref, off by at most err before one rounding to got's type."""
    bound = err * (1 + 2 * HALF_STEP[got.dtype]) + HALF_STEP[got.dtype] * ref.abs()
    d = (got.double().cpu() - ref).abs()
    assert bool((d <= bound).all()), f"{what}: {float((d - bound).max()):.3g} beyond the bound"


def gather(cache, table_row, page_size, num_pages, n):
    """([n, H, D] fp64 of a sequence's first n positions, which of them exist) of a CPU cache [pages, H, slot, D]."""
    t = torch.arange(n)
    page = table_row[torch.div(t, page_size, rounding_mode="floor")].long()
    ok = (page >= 0) & (page < num_pages)
    return cache[page.clamp(0, num_pages - 1), :, t % page_size].double(), ok


def attend(q, kc, vc, table, pos, scale, rotated=None):
    """fp64 attention of q [B, Hq, S, D] over a paged cache (CPU tensors): o, lse and their bounds.
    rotated: (f, scale, interleaved) of the rotation of q.

    Bounds.  A score is a sum of D products of fp32 (or of exact bf16 products): (D + 2) u A, A = scale sum |q k|, and its
    scaling, exponent argument and exp2 4 u (1 + |s|); a bf16 q that is rotated here enters in two bf16 parts, 2^-16 A.
    Twice that for a weight relative to the maximum's, n u for sums of n terms, and 2^-16 for a weight in two
    bf16 parts: relative to sum p |v|.  Finite inputs only reach the rows that see them."""
    B, Hq, S, D = q.shape
    pages, Hkv, ps, _ = kc.shape
    G = Hq // Hkv
    cap = table.shape[1] * ps
    o = torch.zeros(B, Hq, S, D, dtype=torch.float64)
    eo = torch.zeros_like(o)
    lse = torch.full((B, Hq, S), -math.inf, dtype=torch.float64)
    el = torch.zeros_like(lse)
    scale = scale if scale > 0 else 1.0 / math.sqrt(D)
    bf = q.dtype == torch.bfloat16
    for b in range(B):
        n = min(int(pos[b].max()) + 1, cap)
        if n <= 0:
            continue
        k, ok = gather(kc, table[b], ps, pages, n)
        v, _ = gather(vc, table[b], ps, pages, n)
        for s in range(S):
            seen = ok & (torch.arange(n) <= int(pos[b, s]))
            if not bool(seen.any()):
                continue
            ks, vs = k[seen], v[seen]
            m = ks.shape[0]
            qq = q[b, :, s].double()
            if rotated is not None:
                qq, eq = rotate(q[b, :, s], pos[b, s].expand(Hq), *rotated)
                eq = eq + (2.0 ** -16 * qq.abs() if bf else U * qq.abs())
            for h in range(Hq):
                kh, vh = ks[:, h // G], vs[:, h // G]
                x = scale * (kh @ qq[h])
                A = scale * (kh.abs() @ qq[h].abs())
                ds = ((D + 2) * U * A + 4 * U * (1 + x.abs()))
                if rotated is not None:
                    ds = ds + scale * (kh.abs() @ eq[h])
                ds = float(ds.max())
                top = x.max()
                p = torch.exp(x - top)
                L = p.sum()
                o[b, h, s] = p @ vh / L
                lse[b, h, s] = top + torch.log(L)
                el[b, h, s] = ds + (m + 8) * U * (1 + abs(float(lse[b, h, s])))
                eo[b, h, s] = (2 * ds + (2 * m + 8) * U + (2.0 ** -16 if bf else 0.0)) * (p @ vh.abs() / L)
    return o, lse, eo, el


def make_cache(gen, lengths, ps, Hkv, D, dtype, spare=2, wide=None, order="phsd", fill=None):
    """A shuffled pool (CPU) with a page more than the sequences need, `spare` times, and the table.  Slots that no
    sequence holds are `fill` (None: values like the others)."""
    used = [-(-n // ps) if n > 0 else 0 for n in lengths]
    pages = sum(used) + spare
    wide = wide or max(max(used), 1)
    kc = torch.randn(pages, Hkv, ps, D, generator=gen).to(dtype)
    vc = torch.randn(pages, Hkv, ps, D, generator=gen).to(dtype)
    perm = torch.randperm(pages, generator=gen).tolist()
    table = torch.full((len(lengths), wide), -1, dtype=torch.int32)
    free = set(range(pages))
    at = 0
    for b, u in enumerate(used):
        mine = perm[at:at + u]
        at += u
        table[b, :u] = torch.tensor(mine, dtype=torch.int32)
        free -= set(mine)
        if fill is not None and u and lengths[b] % ps:
            kc[mine[-1], :, lengths[b] % ps:] = fill
            vc[mine[-1], :, lengths[b] % ps:] = fill
    if fill is not None:
        for p in free:
            kc[p] = fill
            vc[p] = fill
    return kc, vc, table


def on_gpu(cache, order="phsd"):
    """A CPU cache [pages, H, slot, D] on the GPU, in memory in the given order."""
    if order == "pshd":
        return cache.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    return cache.contiguous().cuda()
