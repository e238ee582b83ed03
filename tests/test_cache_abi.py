"""Host-side checks of include/seer_cache.h and its binding (no GPU needed): exports, sizes and refusals.  Every call
returns from argument validation, which touches no device."""
import ctypes as C
import math
import os
import re

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

from paper_2410_13276_amd import cache, decode  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "seer_cache.h")
FAKE = 0x10000  # aligned, never dereferenced on these paths
ODD = FAKE + 2
INVALID, UNSUPPORTED, WORKSPACE = seer.ERR_INVALID_ARG, seer.ERR_UNSUPPORTED, seer.ERR_WORKSPACE


def test_exports_every_declared_symbol():
    txt = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(seer_[a-z0-9_]+)\s*\(", txt))
    assert names == set(cache.SIGS)
    L = C.CDLL(seer.LIB_PATH)
    for n in names:
        assert hasattr(L, n), n


def test_structures_are_packed_as_declared(tmp_path):
    """Sizes by the C compiler."""
    import shutil
    import subprocess
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no gcc")
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "seer_cache.h"\nint main(void){printf("%zu %zu %zu %zu %zu",sizeof(seer_kv_cache),'
                   'sizeof(seer_kv_tokens),sizeof(seer_kv_queries),sizeof(seer_kv_weight_buf),sizeof(seer_kv_eviction));return 0;}')
    exe = tmp_path / "s"
    subprocess.run([cc, "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [cache._CACHE.size, cache._TOKENS.size, cache._TOKENS.size, cache._WEIGHTS.size, cache._EVICTION.size]


def make_cache(H=2, D=128, dtype=0, group=32, page=16, pages=8, rows=4, wide=4, table=FAKE, ts=4, codes=FAKE, params=FAKE,
               st=None, pst=None, vcodes=FAKE, vparams=FAKE):
    row = D // 2 if group else D
    ng = max(D // group, 1) if group else 1
    st = st or (H * page * row, page * row, row)
    pst = pst or (H * page * ng, page * ng, ng)
    return cache._CACHE.pack(H, D, dtype, group, page, pages, rows, wide, ts, table, codes, params, *st, *pst, vcodes, vparams, *st, *pst)


def tokens(B=2, S=8, dtype=0, reserved=0, H=2, D=128, ks=None, ps=8):
    st = ks or (H * S * D, S * D, D)
    return cache._TOKENS.pack(B, S, dtype, reserved, *st, *st, ps)


def queries(B=2, Hq=4, S=1, dtype=0, H=2, D=128, qs=None, os_=None, ps=8):
    st = (Hq * S * D, S * D, D)
    return cache._TOKENS.pack(B, Hq, S, dtype, *(qs or st), *(os_ or st), ps)


def rope(freq=FAKE, rot=128, inter=0, scale=1.0):
    return decode._ROPE.pack(freq, rot, inter, scale)


CACHE_FAULTS = [
    (dict(H=0), INVALID), (dict(D=0), INVALID), (dict(page=0), INVALID), (dict(pages=0), INVALID), (dict(rows=0), INVALID),
    (dict(wide=0), INVALID), (dict(ts=-1), INVALID), (dict(table=0), INVALID), (dict(table=ODD), INVALID), (dict(codes=0), INVALID),
    (dict(codes=ODD), INVALID), (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED), (dict(group=16), UNSUPPORTED),
    (dict(group=128), UNSUPPORTED), (dict(group=-32), UNSUPPORTED), (dict(params=0), INVALID), (dict(params=FAKE + 4), INVALID),
    (dict(st=(4096, 1024, 40)), UNSUPPORTED), (dict(st=(-4096, 1024, 64)), UNSUPPORTED), (dict(pst=(256, 64, 6)), UNSUPPORTED),
    (dict(page=1 << 20, wide=1 << 11), UNSUPPORTED),
]
VALUE_FAULTS = [(dict(vcodes=0), INVALID), (dict(vcodes=ODD), INVALID), (dict(vparams=0), INVALID)]
WRITTEN_FAULTS = [(dict(st=(4096, 1024, 0)), INVALID), (dict(st=(0, 1024, 64)), INVALID), (dict(pst=(0, 64, 4)), INVALID)]


def append(c, t=tokens(), r=None, k=FAKE, v=FAKE, pos=FAKE, rp=None, rows=None):
    return seer.lib().seer_kv_append_q4(c, t, r, k, v, pos, rp, rows, None)


def read(c, t=tokens(), k=FAKE, v=FAKE, pos=FAKE, rows=None):
    return seer.lib().seer_kv_read(c, t, k, v, pos, rows, None)


def attn(c, t=queries(), r=None, scale=0.0, q=FAKE, pos=FAKE, rp=None, o=FAKE, lse=None, ws=FAKE, nbytes=1 << 30):
    return seer.lib().seer_paged_attn_q4(c, t, r, scale, q, pos, rp, o, lse, ws, nbytes, None)


def weight_buf(win=FAKE, out=FAKE, ins=(2000, 1000), outs=(2000, 1000), width=64, decay=1.0):
    return cache._WEIGHTS.pack(win, out, *ins, *outs, width, decay)


def weigh(c, t=queries(), r=None, scale=0.0, q=FAKE, pos=FAKE, rp=None, lse=FAKE, w=weight_buf()):
    return seer.lib().seer_kv_weights(c, t, r, scale, q, pos, rp, lse, w, None)


def eviction(B=2, keep=10, first=1, last=2, lengths=FAKE, nl=FAKE, nt=FAKE, nts=4, nw=4, width=64, new_width=64, reserved=0,
             w=FAKE, neww=2 * FAKE, st=(128, 64), nst=(128, 64), kept=FAKE):
    return cache._EVICTION.pack(B, keep, first, last, lengths, nl, nt, nts, nw, width, new_width, reserved, w, neww, *st, *nst, kept)


def evict(c, e=eviction(), ws=None, nbytes=0):
    return seer.lib().seer_kv_evict(c, e, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", CACHE_FAULTS)
def test_caches_are_checked(kw, status):
    c = make_cache(**kw)
    for call in (append, read, attn, weigh, evict):
        assert call(c) == status
    assert seer.lib().seer_paged_attn_q4_workspace_bytes(c, queries()) == 0


@pytest.mark.parametrize("kw,status", VALUE_FAULTS)
def test_values_are_checked(kw, status):
    for call in (append, read, attn, evict):
        assert call(make_cache(**kw)) == status


@pytest.mark.parametrize("kw,status", WRITTEN_FAULTS)
def test_written_pools_are_checked(kw, status):
    for call in (append, evict):
        assert call(make_cache(**kw)) == status


def test_caches_of_values_are_checked():
    for call in (read, weigh, evict):
        assert call(make_cache(group=0, dtype=2)) == INVALID
        assert call(make_cache(group=0, st=(4096, 2048, 132))) == UNSUPPORTED
    assert append(make_cache(group=0)) == INVALID and attn(make_cache(group=0)) == INVALID
    assert read(make_cache(group=0, dtype=1)) == INVALID and weigh(make_cache(group=0, dtype=1)) == INVALID
    for call in (append, read, attn, weigh, evict):
        assert call(None) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(t=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(pos=None), INVALID), (dict(k=ODD), INVALID),
    (dict(v=ODD), INVALID), (dict(pos=ODD), INVALID), (dict(rows=ODD), INVALID), (dict(t=tokens(B=0)), INVALID),
    (dict(t=tokens(S=0)), INVALID), (dict(t=tokens(dtype=2)), INVALID), (dict(t=tokens(reserved=1)), INVALID),
    (dict(t=tokens(ps=-1)), INVALID), (dict(t=tokens(B=5)), INVALID), (dict(t=tokens(ks=(2048, 1024, 100))), UNSUPPORTED),
    (dict(t=tokens(ks=(2048, -1024, 128))), UNSUPPORTED), (dict(t=tokens(B=4, S=1 << 26)), UNSUPPORTED)])
def test_tokens_are_checked(kw, status):
    assert append(make_cache(), **kw) == status
    assert read(make_cache(), **kw) == status


def test_more_of_append_and_read():
    c = make_cache()
    assert append(c, rp=ODD) == INVALID
    assert append(c, r=rope(freq=0)) == INVALID and append(c, r=rope(rot=0)) == INVALID and append(c, r=rope(rot=144)) == INVALID
    assert append(c, r=rope(rot=40)) == UNSUPPORTED and append(c, r=rope(inter=2)) == INVALID
    assert append(c, r=rope(scale=math.nan)) == INVALID
    assert read(c, t=tokens(ks=(2048, 0, 128))) == INVALID   # two heads to the same place
    assert append(make_cache(H=65536), t=tokens(H=65536)) == UNSUPPORTED


@pytest.mark.parametrize("kw,status", [
    (dict(t=None), INVALID), (dict(q=None), INVALID), (dict(pos=None), INVALID), (dict(q=ODD), INVALID), (dict(pos=ODD), INVALID),
    (dict(rp=ODD), INVALID), (dict(t=queries(B=0)), INVALID), (dict(t=queries(Hq=0)), INVALID), (dict(t=queries(S=0)), INVALID),
    (dict(t=queries(Hq=3)), INVALID), (dict(t=queries(dtype=3)), INVALID), (dict(t=queries(ps=-1)), INVALID),
    (dict(t=queries(B=5)), INVALID), (dict(t=queries(qs=(512, 128, 4))), UNSUPPORTED), (dict(scale=math.nan), INVALID),
    (dict(scale=math.inf), INVALID), (dict(scale=2.0 ** 101), INVALID), (dict(r=rope(rot=24)), UNSUPPORTED),
    (dict(r=rope(freq=0)), INVALID), (dict(t=queries(Hq=2, H=2, S=(1 << 23) + 1, qs=(0, 0, 0), os_=(1 << 40, 1 << 38, 128))), UNSUPPORTED)])
def test_queries_are_checked(kw, status):
    assert attn(make_cache(), **kw) == status
    assert weigh(make_cache(), **kw) == status


def test_more_of_attention():
    many = queries(B=64, Hq=2 * 1024, S=4096, qs=(0, 0, 0), os_=(1 << 40, 1 << 30, 128))  # 2^25 blocks of 16 rows
    assert attn(make_cache(rows=64), t=many) == UNSUPPORTED and weigh(make_cache(rows=64), t=many) == UNSUPPORTED
    c = make_cache()
    assert attn(c, o=None) == INVALID and attn(c, o=ODD) == INVALID and attn(c, lse=ODD) == INVALID
    assert attn(c, t=queries(os_=(512, 0, 128))) == INVALID
    assert attn(c, ws=None) == WORKSPACE and attn(c, ws=FAKE + 16) == INVALID
    need = seer.lib().seer_paged_attn_q4_workspace_bytes(c, queries())
    # 2 parts a workgroup of 4 rows (4 groups share the 16 columns): maximum and sum, and 128 sums; a record for each pair
    assert need == 256 + 2 * 512 * 4 * 8 + 2 * 512 * 4 * 128 * 4
    assert attn(c, t=queries(), nbytes=need - 1) == WORKSPACE


def test_more_of_weights():
    c = make_cache()
    assert weigh(c, lse=None) == INVALID and weigh(c, lse=ODD) == INVALID and weigh(c, w=None) == INVALID
    for kw in (dict(out=0), dict(out=ODD), dict(win=ODD), dict(win=0), dict(width=0), dict(decay=math.nan), dict(decay=math.inf),
               dict(ins=(-1, 0)), dict(outs=(-1, 64)), dict(outs=(128, 63)), dict(outs=(0, 64)), dict(ins=(2000, 500))):
        assert weigh(c, w=weight_buf(**kw)) == INVALID, kw


def test_more_of_eviction():
    c = make_cache()
    assert evict(c, None) == INVALID
    for kw in (dict(B=0), dict(B=5), dict(keep=0), dict(first=-1), dict(last=-1), dict(first=8, last=3), dict(lengths=0),
               dict(nl=0), dict(nt=0), dict(w=0), dict(neww=0), dict(kept=0), dict(lengths=ODD), dict(kept=ODD), dict(nw=0),
               dict(keep=65, new_width=65), dict(new_width=9), dict(width=0), dict(reserved=1), dict(neww=FAKE), dict(st=(-1, 64)),
               dict(nst=(128, 63)), dict(nst=(0, 64)), dict(nts=-1)):
        assert evict(c, eviction(**kw)) == INVALID, kw
    long_rows = make_cache(page=64, wide=1024)
    need = seer.lib().seer_kv_evict_workspace_bytes(long_rows, 2)
    assert need == 2 * 2 * 4 * (3 * 2048 + 64) * 4 and seer.lib().seer_kv_evict_workspace_bytes(c, 2) == 0  # 4 parts of 16384 slots
    assert evict(long_rows) == WORKSPACE and evict(long_rows, ws=FAKE, nbytes=need - 1) == WORKSPACE
    assert evict(long_rows, ws=FAKE + 128, nbytes=need) == INVALID
    big = make_cache(H=65535, rows=100)
    assert evict(big, eviction(B=100, st=(0, 0), nst=(1 << 30, 64))) == UNSUPPORTED


# ---------------------------------------------------------------------------
# the binding's own checks: tensors on the CPU
# ---------------------------------------------------------------------------

def test_binding_refuses_cpu_tensors():
    kc, vc = seer.alloc_kv_cache_q4(4, 16, 2, 64, device="cpu")
    k = torch.zeros(3, 2, 64)
    pos = torch.zeros(3, dtype=torch.int32)
    table = torch.zeros(3, 1, dtype=torch.int32)
    lse, w = torch.zeros(3, 2), torch.zeros(3, 2, 16)
    for call in (lambda: seer.kv_append_q4(k, k, kc, vc, table, pos), lambda: seer.kv_read(kc, vc, table, pos),
                 lambda: seer.paged_attn_q4(k, kc, vc, table, pos), lambda: seer.kv_weights(k, kc, table, pos, lse, w),
                 lambda: seer.kv_evict(kc, vc, table, pos, w, table, 4)):
        with pytest.raises(ValueError):
            call()


def test_pools_are_described():
    kc, vc = seer.alloc_kv_cache_q4(4, 16, 2, 128, group=64, device="cpu")
    assert kc.head_dim == 128 and kc.group == 64 and vc.codes.shape == (4, 2, 16, 64) and vc.params.shape == (4, 2, 16, 2, 2)
    with pytest.raises(ValueError):
        seer.alloc_kv_cache_q4(4, 16, 2, 128, group=16, device="cpu")
    with pytest.raises(ValueError):
        seer.alloc_kv_cache_q4(4, 16, 2, 96, group=64, device="cpu")


def test_pools_are_checked():
    kc, _ = seer.alloc_kv_cache_q4(4, 16, 2, 128, device="cpu")
    assert seer.Q4Pool(kc.codes.transpose(1, 2), kc.params.transpose(1, 2)).shape == (4, 16, 2, 128)
    for codes, params in ((kc.codes.to(torch.int8), kc.params), (kc.codes, kc.params.to(torch.float16))):
        with pytest.raises(TypeError):
            seer.Q4Pool(codes, params)
    for codes, params in ((kc.codes[0], kc.params), (kc.codes, kc.params[..., 0]), (kc.codes, kc.params[:3]),
                          (kc.codes.transpose(2, 3), kc.params.transpose(2, 3)), (kc.codes, kc.params.transpose(3, 4)),
                          (kc.codes[..., ::2], kc.params), (kc.codes, kc.params[..., :1, :1])):
        with pytest.raises(ValueError):
            seer.Q4Pool(codes, params)


def test_a_pool_keeps_its_tensors():
    kc, _ = seer.alloc_kv_cache_q4(4, 16, 2, 64, device="cpu")
    for name, value in (("codes", kc.codes), ("params", kc.params), ("group", 64)):
        with pytest.raises(AttributeError):
            setattr(kc, name, value)
