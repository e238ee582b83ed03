"""The operators that carry a prompt on to generation, as cases that can be timed and checked:

    rope        rotary positions of Q and K (and their gradient), between the gate and the attention
    append      keys and values of new tokens into a paged cache, the keys rotated on the way
    attend      attention of new tokens over that cache

    own                    False: the plain form, in 32 bits (angles in 64); True: the package's calls
    listed(), draw(rng)    the named cases, and one more of the same ranges
    prepare(case, seed)    what a program has in hand before the call, drawn on the GPU
    run(state)             one pass; returns its outputs
    work(case)             bytes and operations one pass cannot do without
    exact(case, seed)      the outputs in 64 bits, from the definitions
"""
import math
import random

import torch

own = False

PROMPTS = [1900, 37, 512, 845, 128, 3300, 260, 77, 1024, 6100, 400, 15, 2222, 690, 1500, 64, 333, 4500, 980, 200]


def _text(lengths):
    return ",".join(str(n) for n in lengths)


def _numbers(text):
    return [int(x) for x in text.split(",")]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _rope(name, dtype, batch, hq, hkv, dim, seq, rot, interleaved=False, scaling="none", layout="bhsd",
          grad=False, positions="start"):
    """positions: "start" (token s of a row is at start + s) or "each" (a tensor, rows beginning anywhere)."""
    c = dict(kind="rope", dtype=dtype, batch=batch, hq=hq, hkv=hkv, dim=dim, seq=seq, rot=rot, interleaved=interleaved,
             scaling=scaling, layout=layout, grad=grad, positions=positions)
    return dict(name=name, **c) if name else c


def _append(name, dtype, hkv, dim, page, rot, new, before, packed, interleaved=False, scaling="none", order="phsd"):
    """new: tokens added to each sequence, before: tokens that it already holds.  packed: the new tokens stand back to
    back, [tokens, heads, dim]; otherwise they are padded to [batch, heads, longest, dim].  rot 0: no rotation.  order: the
    cache's memory order, head before slot ("phsd") or slot before head ("pshd")."""
    c = dict(kind="append", dtype=dtype, hkv=hkv, dim=dim, page=page, rot=rot, new=_text(new), before=_text(before),
             packed=packed, interleaved=interleaved, scaling=scaling, order=order)
    return dict(name=name, **c) if name else c


def _attend(name, dtype, hq, hkv, dim, page, lengths, tokens=1, rot=0, interleaved=False, scaling="none", order="phsd",
            lse=False):
    """lengths: keys that each sequence's last new token sees; tokens: new tokens per sequence.  rot 0: q comes rotated."""
    c = dict(kind="attend", dtype=dtype, hq=hq, hkv=hkv, dim=dim, page=page, lengths=_text(lengths), tokens=tokens, rot=rot,
             interleaved=interleaved, scaling=scaling, order=order, lse=lse)
    return dict(name=name, **c) if name else c


def listed():
    mixed = random.Random(3)
    return [
        # the smallest configuration (fp32, 2 / 1 heads of 64): launch and latency decide
        _rope("rope_f32_s1k", "f32", 1, 2, 1, 64, 1024, 64),
        # a prompt of the benchmark's 8k workload, frequencies scaled in bands for a long context
        _rope("rope_s8k", "bf16", 1, 32, 8, 128, 8192, 128, scaling="bands"),
        # a batch of odd length of a small model that rotates half of each head in adjacent pairs, token-major as a
        # projection leaves it, its rows at positions of their own
        _rope("rope_part_b4_s4001", "bf16", 4, 16, 4, 64, 4001, 32, interleaved=True, scaling="yarn", layout="bshd",
              positions="each"),
        # the way back through the rotation in a training step at 32k
        _rope("rope_grad_s32k", "bf16", 1, 32, 8, 128, 32768, 128, grad=True),
        # one decode step of a server: a token for each of 64 sequences
        _append("append_b64_t1", "bf16", 8, 128, 16, 128, [1] * 64, [_log(mixed, 50, 1000) for _ in range(64)], True),
        # the prompts of a server's batch, packed, into empty caches
        _append("append_prompts_20", "bf16", 8, 128, 64, 128, PROMPTS, [0] * 20, True, scaling="bands"),
        # fp32, chunks of unequal length padded to the longest, pages of no power of two, half of the head rotated
        _append("append_f32_b3_page24", "f32", 4, 64, 24, 32, [700, 1, 333], [100, 1001, 23], False, interleaved=True,
                order="pshd"),
        # the smallest decode step (fp32, 2 / 1 heads of 64)
        _attend("attend_f32_b1_s1k", "f32", 2, 1, 64, 16, [1000]),
        # a chat answer's token, one sequence: too little work to fill the GPU
        _attend("attend_b1_s2k", "bf16", 32, 8, 128, 16, [2047], rot=128),
        # a token after the benchmark's 128k prompt
        _attend("attend_b1_s128k", "bf16", 32, 8, 128, 64, [131072], rot=128, scaling="bands", lse=True),
        # a server's batch of unequal lengths
        _attend("attend_b64_mixed", "bf16", 32, 8, 128, 16, [_log(mixed, 200, 16384) for _ in range(64)], rot=128),
        # four drafted tokens to be verified, 28 / 4 heads, token-major cache
        _attend("attend_draft4_b8", "bf16", 28, 4, 128, 128, [30011, 4500, 15000, 700, 22022, 9001, 64, 12345], tokens=4,
                order="pshd", lse=True),
    ]


def draw(rng):
    hq, hkv, dim = rng.choice([(2, 1, 64), (8, 2, 128), (16, 4, 64), (32, 8, 128), (32, 8, 128), (28, 4, 128), (12, 12, 64),
                               (24, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    size = dim * (4 if dtype == "f32" else 2)
    how = dict(interleaved=rng.random() < 0.4, scaling=rng.choice(["none", "linear", "bands", "yarn"]))
    rot = rng.choice([dim, dim, dim // 2, 16, dim - 16])
    kind = rng.choice(["rope", "append", "attend", "attend"])
    if kind == "rope":
        batch = rng.randint(1, 4)
        most = min(40000, (300 << 20) // ((hq + hkv) * size * batch))  # 300 MiB in, 300 out
        return _rope(None, dtype, batch, hq, hkv, dim, _log(rng, 1, most), rot, layout=rng.choice(["bhsd", "bshd"]),
                     grad=rng.random() < 0.3, positions=rng.choice(["start", "each"]), **how)
    page = rng.choice([8, 16, 16, 24, 32, 64, 128, 256, rng.randint(1, 100)])
    order = rng.choice(["phsd", "pshd"])
    if rng.random() < 0.2:
        rot = 0
    if kind == "append":
        count = _log(rng, 1, 128)
        most = min(8192, (48 << 20) // (hkv * size * count))
        new = [1] * count if rng.random() < 0.4 else [_log(rng, 1, most) for _ in range(count)]
        return _append(None, dtype, hkv, dim, page, rot, new, [_log(rng, 1, 2000) - 1 for _ in new], rng.random() < 0.6,
                       order=order, **how)
    count = _log(rng, 1, 96)
    most = min(131072, (900 << 20) // (2 * hkv * size * count))
    lengths = [max(4, _log(rng, 1, most)) for _ in range(count)]
    return _attend(None, dtype, hq, hkv, dim, page, lengths, tokens=rng.choice([1, 1, 1, 2, 4]), rot=rot, order=order,
                   lse=rng.random() < 0.4, **how)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _frequencies(rot, scaling):
    """Angles per position of the rot / 2 planes (fp64, on the GPU) and the factor on the rotated values: base 500000,
    and for a context 8 times that of training either all angles divided by 8 ("linear"), those of wavelengths beyond
    the trained context with a ramp ("bands"), or a ramp over the planes' turns with a factor ("yarn")."""
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    turns = 8192 * f / (2 * math.pi)
    if scaling == "linear":
        return f / 8, 1.0
    if scaling == "bands":
        keep = ((turns - 1) / 3).clamp(0, 1)
        return f * (keep + (1 - keep) / 8), 1.0
    if scaling == "yarn":
        keep = (torch.log2(turns.clamp_min(1e-30)) / 5).clamp(0, 1)
        return f * (keep + (1 - keep) / 8), 0.1 * math.log(8) + 1
    return f, 1.0


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    return torch.randn(shape, generator=g, device="cuda", dtype=dt) * scale


def _heads(g, case, batch, heads, seq, scale=1.0):
    """[batch, heads, seq, dim], in memory head-major or token-major."""
    if case.get("layout") == "bshd":
        return _normal(g, (batch, seq, heads, case["dim"]), case["dtype"], scale).transpose(1, 2)
    return _normal(g, (batch, heads, seq, case["dim"]), case["dtype"], scale)


def _cache(g, case, held):
    """A pool of pages in no order, the table of each sequence's pages (-1 past them), for sequences of `held` tokens."""
    page, hkv, dim = case["page"], case["hkv"], case["dim"]
    used = [-(-n // page) for n in held]
    pool = sum(used) + 3
    shape = (pool, page, hkv, dim) if case["order"] == "pshd" else (pool, hkv, page, dim)
    kc, vc = _normal(g, shape, case["dtype"]), _normal(g, shape, case["dtype"])
    if case["order"] == "pshd":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    wide = max(used) + 5  # a table has room for longer sequences than there are
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    ends = torch.tensor(used, device="cuda").cumsum(0)[:, None]
    col = torch.arange(wide, device="cuda")[None, :]
    n = torch.tensor(used, device="cuda")[:, None]
    table = torch.where(col < n, order[(ends - n + col).clamp(max=pool - 1)], -1).to(torch.int32)
    return kc, vc, table.contiguous()


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    s["freqs"], s["scale"] = _frequencies(case["rot"], case["scaling"])
    if case["kind"] == "rope":
        b, n = case["batch"], case["seq"]
        s["q"], s["k"] = _heads(g, case, b, case["hq"], n), _heads(g, case, b, case["hkv"], n)
        s["start"] = 0
        s["positions"] = None
        if case["positions"] == "each":
            first = torch.randint(0, 60000, (b, 1), generator=g, device="cuda")
            s["positions"] = (first + torch.arange(n, device="cuda")).to(torch.int32)
        return s
    if case["kind"] == "append":
        new, before = _numbers(case["new"]), _numbers(case["before"])
        s["kc"], s["vc"], s["table"] = _cache(g, case, [a + b for a, b in zip(new, before)])
        ends = torch.tensor(new, device="cuda").cumsum(0)
        begin = torch.tensor(before, device="cuda")
        count = torch.tensor(new, device="cuda")
        if case["packed"]:
            t = sum(new)
            row = torch.searchsorted(ends, torch.arange(t, device="cuda"), right=True)
            s["positions"] = (begin[row] + torch.arange(t, device="cuda") - (ends - count)[row]).to(torch.int32)
            s["rows"] = row.to(torch.int32)
            s["k"], s["v"] = (_normal(g, (t, case["hkv"], case["dim"]), case["dtype"]) for _ in range(2))
        else:
            col = torch.arange(max(new), device="cuda")[None, :]
            s["positions"] = torch.where(col < count[:, None], begin[:, None] + col, -1).to(torch.int32)
            s["rows"] = None
            s["k"], s["v"] = (_normal(g, (len(new), case["hkv"], max(new), case["dim"]), case["dtype"]) for _ in range(2))
        # the tokens that are none of the padding, as a scheduler that pads a batch knows them
        s["real"] = (s["positions"].reshape(-1) >= 0).nonzero()[:, 0]
        return s
    lengths = _numbers(case["lengths"])
    t = case["tokens"]
    s["longest"] = max(lengths)
    s["kc"], s["vc"], s["table"] = _cache(g, case, lengths)
    s["q"] = _normal(g, (len(lengths), case["hq"], t, case["dim"]), case["dtype"], 1.5)
    last = torch.tensor(lengths, device="cuda")[:, None]
    s["positions"] = (last - t + torch.arange(t, device="cuda")[None, :]).to(torch.int32).contiguous()
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _turned(x, positions, freqs, scale, interleaved, back=False):
    """x [.., dim] rotated at positions (which broadcast over x's leading axes), in 32 bits with 64-bit angles."""
    rot = 2 * freqs.numel()
    a = positions.double().unsqueeze(-1) * freqs
    c, n = (a.cos() * scale).float(), (a.sin() * (-scale if back else scale)).float()
    y = x.float()
    if interleaved:
        u, w = y[..., 0:rot:2], y[..., 1:rot:2]
        z = torch.stack((u * c - w * n, u * n + w * c), -1).flatten(-2)
    else:
        u, w = y[..., :rot // 2], y[..., rot // 2:rot]
        z = torch.cat((u * c - w * n, u * n + w * c), -1)
    return torch.cat((z, y[..., rot:]), -1)


def _rope_plain(s):
    case = s["case"]
    at = s["positions"]
    if at is None:
        at = s["start"] + torch.arange(case["seq"], device="cuda")[None, :]
    how = (at[:, None, :], s["freqs"], s["scale"], case["interleaved"], case["grad"])
    return {"q": _turned(s["q"], *how).to(s["q"].dtype), "k": _turned(s["k"], *how).to(s["k"].dtype)}


def _append_plain(s):
    case = s["case"]
    at = s["positions"]
    if case["packed"]:
        k, v, row = s["k"], s["v"], s["rows"].long()
    else:
        k, v = (s[x].transpose(1, 2).reshape(-1, case["hkv"], case["dim"]) for x in "kv")
        row = torch.arange(at.shape[0], device="cuda").repeat_interleave(at.shape[1])
    real = s["real"]
    at, row = at.reshape(-1)[real].long(), row[real]
    k, v = k[real], v[real]
    if case["rot"]:
        k = _turned(k, at[:, None], s["freqs"], s["scale"], case["interleaved"]).to(k.dtype)
    page = s["table"][row, at // case["page"]].long()
    s["kc"][page, :, at % case["page"]] = k
    s["vc"][page, :, at % case["page"]] = v
    return {"k": s["kc"], "v": s["vc"]}


def _attend_plain(s):
    case = s["case"]
    b, hq, t, dim = s["q"].shape
    hkv = case["hkv"]
    q = s["q"].float()
    if case["rot"]:
        q = _turned(s["q"], s["positions"][:, None, :], s["freqs"], s["scale"], case["interleaved"])
    u = torch.arange(s["longest"], device="cuda")
    page = s["table"][:, u // case["page"]].clamp_min(0).long()
    k = s["kc"][page, :, u % case["page"]].float().permute(0, 2, 3, 1).contiguous()  # [b, hkv, dim, keys]
    x = torch.matmul(q.reshape(b, hkv, -1, dim), k).reshape(b, hkv, hq // hkv, t, -1) / math.sqrt(dim)
    del k
    x = x.masked_fill(u > s["positions"][:, None, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    v = s["vc"][page, :, u % case["page"]].float().permute(0, 2, 1, 3).contiguous()  # [b, hkv, keys, dim]
    o = torch.matmul(p.reshape(b, hkv, -1, p.shape[-1]), v).reshape(b, hkv, hq // hkv, t, dim)
    o = torch.where(total > 0, o / total, 0.0).reshape(b, hq, t, dim).to(s["q"].dtype)
    out = {"o": o}
    if case["lse"]:
        out["lse"] = (m + torch.log(total)).reshape(b, hq, t)
    return out


def _call(s):
    import paper_2410_13276_amd as seer
    case = s["case"]
    how = dict(inv_freq=s["freqs"], interleaved=case["interleaved"], rope_scale=s["scale"]) if case["rot"] else {}
    if case["kind"] == "rope":
        f = seer.rope_grad if case["grad"] else seer.rope
        q, k = f(s["q"], s["k"], positions=s["positions"], start=s["start"], **how)
        return {"q": q, "k": k}
    if case["kind"] == "append":
        seer.kv_append(s["k"], s["v"], s["kc"], s["vc"], s["table"], s["positions"], rows=s["rows"], **how)
        return {"k": s["kc"], "v": s["vc"]}
    o, lse = seer.paged_attn(s["q"], s["kc"], s["vc"], s["table"], s["positions"], want_lse=case["lse"], **how)
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}


def run(s):
    if own:
        return _call(s)
    kind = s["case"]["kind"]
    return _rope_plain(s) if kind == "rope" else _append_plain(s) if kind == "append" else _attend_plain(s)


# ---------------------------------------------------------------------------
# what one pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    size = case["dim"] * (4 if case["dtype"] == "f32" else 2)
    if case["kind"] == "rope":
        rows = case["batch"] * case["seq"]
        heads = case["hq"] + case["hkv"]
        each = 4.0 * rows if case["positions"] == "each" else 0.0
        return {"bytes": 2.0 * rows * heads * size + each, "flops": 3.0 * rows * heads * case["rot"]}
    if case["kind"] == "append":
        rows = sum(_numbers(case["new"]))
        return {"bytes": rows * (4.0 * case["hkv"] * size + 12.0), "flops": 3.0 * rows * case["hkv"] * case["rot"]}
    lengths, t = _numbers(case["lengths"]), case["tokens"]
    keys = sum(lengths)
    seen = sum(n - t + 1 + i for n in lengths for i in range(t))
    rows = len(lengths) * t * case["hq"]
    nbytes = 2.0 * keys * case["hkv"] * size + 2.0 * rows * size + (4.0 * rows if case["lse"] else 0.0)
    nbytes += sum(4.0 * -(-n // case["page"]) for n in lengths)
    return {"bytes": nbytes, "flops": 4.0 * case["hq"] * case["dim"] * seen}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _rotation(x, positions, freqs, scale, interleaved, back):
    """x as complex numbers, one per plane, times scale exp(+-i position f)."""
    half = freqs.numel()
    y = x.double()
    a, b = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if interleaved else (y[..., :half], y[..., half:2 * half])
    angle = positions.double().unsqueeze(-1) * freqs
    z = torch.complex(a, b) * torch.polar(torch.full_like(angle, scale), -angle if back else angle)
    out = y.clone()
    if interleaved:
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = z.real, z.imag
    else:
        out[..., :half], out[..., half:2 * half] = z.real, z.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    turn = (s["freqs"], s["scale"], case["interleaved"])
    if case["kind"] == "rope":
        at = s["positions"]
        if at is None:
            at = torch.arange(s["start"], s["start"] + case["seq"], device="cuda").expand(case["batch"], -1)
        return {x: _rotation(s[x], at.unsqueeze(1), *turn, case["grad"]) for x in "qk"}
    page = case["page"]
    if case["kind"] == "append":
        kc, vc = s["kc"].double(), s["vc"].double()
        done = 0
        for row, (n, first) in enumerate(zip(_numbers(case["new"]), _numbers(case["before"]))):
            k, v = ((s[x][done:done + n] if case["packed"] else s[x][row, :, :n].transpose(0, 1)) for x in "kv")
            done += n
            at = torch.arange(first, first + n, device="cuda")
            where = s["table"][row].long()[torch.div(at, page, rounding_mode="floor")]
            kc[where, :, at % page] = _rotation(k, at.unsqueeze(1), *turn, False) if case["rot"] else k.double()
            vc[where, :, at % page] = v.double()
        return {"k": kc, "v": vc}
    b, hq, t, dim = s["q"].shape
    hkv = case["hkv"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(b, hq, t, dtype=torch.float64, device="cuda")
    for row, n in enumerate(_numbers(case["lengths"])):
        pages = s["table"][row, :-(-n // page)].long()
        k, v = (s[x][pages].transpose(0, 1).reshape(hkv, -1, dim)[:, :n].double() for x in ("kc", "vc"))
        q = s["q"][row].double()
        at = torch.arange(n - t, n, device="cuda")
        if case["rot"]:
            q = _rotation(q, at, *turn, False)
        g = hq // hkv
        x = torch.matmul(q.reshape(hkv, g * t, dim), k.transpose(1, 2).contiguous()) / math.sqrt(dim)
        x = x.reshape(hkv, g, t, n).masked_fill(torch.arange(n, device="cuda") > at[:, None], -math.inf)
        total = torch.logsumexp(x, -1, keepdim=True)
        o[row] = torch.matmul(torch.exp(x - total).reshape(hkv, g * t, n), v).reshape(hq, t, dim)
        lse[row] = total.reshape(hq, t)
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}
