"""The bounds of cache_tight hold for the arithmetic that the calls over 4 bits state, formed here in fp32 on the CPU, and not for it with a part left out."""
import math

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")

import cache_ref as R  # noqa: E402
import cache_tight as T  # noqa: E402
from decode_ref import freqs, rotate  # noqa: E402


def parts_of(x, n):
    """fp32 x as n bf16 parts: three hold it exactly, fewer are rounded to nearest."""
    out = []
    for _ in range(n):
        y = x.to(torch.bfloat16).float()
        out.append(y)
        x = x - y
    return out


def chain(terms, start):
    for i in range(terms.shape[-1]):
        start = start + terms[..., i]
    return start


def tree(x):
    """Sums of the last axis (a power of two) in pairs."""
    while x.shape[-1] > 1:
        x = x[..., ::2] + x[..., 1::2]
    return x


def products(a_parts, u, start):
    """start + sum over the last axis of a u in fp32, least parts first, 32 products (an instruction's) at a time in pairs."""
    for a in reversed(a_parts):
        y = a * u
        y = torch.nn.functional.pad(y, (0, -y.shape[-1] % 32))
        start = chain(tree(y.reshape(*y.shape[:-1], -1, 32))[..., 0], start)
    return start


def entering(c, centred):
    """Codes [.., D] as they enter, (+-1 and the number), and what of 1 + 7.5 / 16 has to come out again."""
    sign = torch.where(torch.arange(c.shape[-1]) % 8 < 4, 1.0, -1.0)
    u = 1.0 + torch.where(sign > 0, c, 15 - c).float() / 16
    return sign, u - 1.5 if centred else u, 1.46875 - (1.5 if centred else 0.0)


def scores(c, step, mid, q, scale, centred, parts):
    """Of rows q [r, D] with keys [n, ..]: [r, n], unscaled / 16."""
    sign, u, out = entering(c, centred)
    ng = step.shape[-1]
    g = c.shape[-1] // ng
    s = torch.zeros(q.shape[0], c.shape[0])
    for i in range(ng):
        at = slice(g * i, g * i + g)
        signed = (q * sign)[:, None, at]
        y = products(parts_of(signed, parts), u[None, :, at], -out * tree(signed)[..., 0])
        s = s + mid[:, i].float() * tree(q[:, at]) / 16
        s = s + step[:, i].float() * y
    return s


def emulate(q, kpool, vpool, table, page, pos, turn, centred, q_parts, p_parts, drop=None):
    """o and lse [B, Hq, S, ..] of the stated arithmetic in fp32."""
    B, Hq, S, D = q.shape
    pools = [R.opened(p) for p in (kpool, vpool)]
    Hkv = pools[0][0].shape[1]
    o, lse = torch.zeros(B, Hq, S, D), torch.zeros(B, Hq, S)
    scale = torch.tensor(16.0 * 1.4426950408889634 / math.sqrt(D), dtype=torch.float32)
    for b in range(B):
        for s in range(S):
            n = int(pos[b, s]) + 1
            for h in range(Hq):
                (c, st, mi), (cv, sv, mv) = (tuple(R.rows_of(x, table[b], page, n)[:, h // (Hq // Hkv)] for x in p) for p in pools)
                x = q[b, h, s].float() if turn is None else rotate(q[b, h, s], pos[b, s], *turn)[0].float()
                y = scores(c, st, mi, x[None], scale, centred, q_parts)[0]
                p = torch.exp2((y - y.max()) * scale)
                if drop is not None:
                    p[drop] = 0.0
                lse[b, h, s] = (y.max() * scale + torch.log2(p.sum())) * math.log(2.0)
                g = D // st.shape[-1]
                for d0 in range(0, D, g):
                    i = d0 // g
                    u = 1.0 + cv[:, d0:d0 + g].float() / 16 - (1.5 if centred else 0.0)
                    sign = torch.where(torch.arange(n) % 8 < 4, 1.0, -1.0)
                    u = torch.where(sign[:, None] > 0, u, (1.0 + (15 - cv[:, d0:d0 + g]).float() / 16) - (1.5 if centred else 0.0))
                    w = parts_of(p * sv[:, i].float() * sign, p_parts)
                    out = 1.46875 - (1.5 if centred else 0.0)
                    total = torch.zeros(g)
                    for t in range(0, n, 64):
                        y0 = torch.zeros(g)
                        for part in reversed(w):
                            y0 = chain(torch.full((g, 1), -out) * part[None, t:t + 64], y0)
                        total = total + products([part[None, t:t + 64] for part in w], u[t:t + 64].T, y0)
                    o[b, h, s, d0:d0 + g] = (16 * total + chain((p * mv[:, i].float())[None], torch.zeros(1))) / p.sum()
    return o.to(q.dtype), lse


CASES = [(2, 1, 64, 32), (2, 1, 64, 64), (8, 2, 128, 32), (8, 2, 128, 64)]
RIGHT = {torch.float32: (True, 3, 3), torch.bfloat16: (False, 3, 2)}


def call(gen, dtype, Hq, Hkv, D, group, pool, lengths, turn):
    table, pages, _ = R.paged(gen, lengths, 16)
    kc, vc = (pool(seer, gen, pages, Hkv, 16, D, group, device="cpu") for _ in range(2))
    q = (1.5 * torch.randn(len(lengths), Hq, 1, D, generator=gen)).to(dtype)
    pos = torch.tensor(lengths, dtype=torch.int32)[:, None] - 1
    return q, kc, vc, table, 16, pos, turn


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pool", [T.random_pool, T.outlier_pool])
@pytest.mark.parametrize("Hq,Hkv,D,group", CASES)
def test_the_stated_arithmetic(dtype, pool, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(Hq + D + group)
    q, kc, vc, table, page, pos, turn = call(gen, dtype, Hq, Hkv, D, group, pool, [1, 2, 3, 70], (freqs(D, 500000.0), 1.0, False))
    T.check(*emulate(q, kc, vc, table, page, pos, turn, *RIGHT[dtype]), T.attend(q, kc, vc, table, page, pos, 0.0, turn), "right")


def wrong(what, dtype):
    centred, q_parts, p_parts = RIGHT[dtype]
    return {"uncentred": (False, q_parts, p_parts), "q in two": (centred, 2, p_parts), "q in one": (centred, 1, p_parts),
            "p in one": (centred, q_parts, 1), "p in two": (centred, q_parts, 2), "a key": (centred, q_parts, p_parts, -1)}[what]


@pytest.mark.parametrize("dtype,pool,what,lengths", [
    (torch.float32, T.outlier_pool, "uncentred", [70]),
    (torch.float32, T.random_pool, "q in two", [1, 2, 1, 3]),
    (torch.float32, T.random_pool, "q in one", [70]),
    (torch.float32, T.random_pool, "p in two", [70]),
    (torch.float32, T.random_pool, "a key", [300]),
    (torch.bfloat16, T.random_pool, "q in one", [1, 2, 1, 3]),
    (torch.bfloat16, T.random_pool, "p in one", [70]),
    (torch.bfloat16, T.random_pool, "a key", [300]),
])
@pytest.mark.parametrize("Hq,Hkv,D,group", CASES)
def test_a_part_left_out(dtype, pool, what, lengths, Hq, Hkv, D, group):
    gen = torch.Generator().manual_seed(Hq + D + group)
    q, kc, vc, table, page, pos, turn = call(gen, dtype, Hq, Hkv, D, group, pool, lengths, (freqs(D, 500000.0), 1.0, False))
    got = emulate(q, kc, vc, table, page, pos, turn, *wrong(what, dtype))
    with pytest.raises(AssertionError):
        T.check(*got, T.attend(q, kc, vc, table, page, pos, 0.0, turn), what)
