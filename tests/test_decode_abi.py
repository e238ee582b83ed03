"""Host-side checks of include/seer_decode.h and its binding (no GPU needed): exports, sizes and
refusals.  Every call returns from argument validation, which touches no device."""
import ctypes as C
import math
import os
import re

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

from paper_2410_13276_amd import decode  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "seer_decode.h")
FAKE = 0x10000  # aligned, never dereferenced on these paths
ODD = FAKE + 2


def test_exports_every_declared_symbol():
    txt = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(seer_[a-z_]+)\s*\(", txt))
    assert names == set(decode.SIGS)
    L = C.CDLL(seer.LIB_PATH)
    for n in names:
        assert hasattr(L, n), n


def rope_params(freq=FAKE, rot=128, inter=0, scale=1.0):
    return decode._ROPE.pack(freq, rot, inter, scale)


def rope_call(B=1, Hq=4, Hkv=2, S=64, D=128, dtype=0, params=rope_params(), q=FAKE, k=FAKE, qo=FAKE, ko=FAKE,
              positions=None, start=0, qs=None, qos=None, pos_stride=0, desc=True):
    st = lambda H: (H * S * D, S * D, D)
    d = decode._ROPE_DESC.pack(B, Hq, Hkv, S, D, dtype, *(qs or st(Hq)), *st(max(Hkv, 0)), *(qos or st(Hq)),
                               *st(max(Hkv, 0)), pos_stride)
    return seer.lib().seer_rope(d if desc else None, params, q, k, qo, ko, positions, start, 0, None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=False), seer.ERR_INVALID_ARG),
    (dict(params=None), seer.ERR_INVALID_ARG),
    (dict(q=None), seer.ERR_INVALID_ARG),
    (dict(qo=None), seer.ERR_INVALID_ARG),
    (dict(k=None), seer.ERR_INVALID_ARG),           # heads_kv 2, but no K
    (dict(Hkv=0), seer.ERR_INVALID_ARG),            # a K without heads
    (dict(Hkv=-1, k=None, ko=None), seer.ERR_INVALID_ARG),
    (dict(ko=None), seer.ERR_INVALID_ARG),
    (dict(B=0), seer.ERR_INVALID_ARG),
    (dict(S=0), seer.ERR_INVALID_ARG),
    (dict(Hq=0), seer.ERR_INVALID_ARG),
    (dict(dtype=2), seer.ERR_INVALID_ARG),
    (dict(D=96), seer.ERR_UNSUPPORTED),
    (dict(D=256), seer.ERR_UNSUPPORTED),
    (dict(q=ODD), seer.ERR_INVALID_ARG),
    (dict(ko=ODD), seer.ERR_INVALID_ARG),
    (dict(positions=ODD + 1), seer.ERR_INVALID_ARG),
    (dict(qs=(0, 0, 132)), seer.ERR_UNSUPPORTED),    # no multiple of 8 bf16
    (dict(qs=(-128, 0, 128)), seer.ERR_UNSUPPORTED),
    (dict(qos=(0, 0, 128)), seer.ERR_INVALID_ARG),   # four heads written to one place
    (dict(pos_stride=-1), seer.ERR_INVALID_ARG),
    (dict(start=2 ** 31 - 63), seer.ERR_INVALID_ARG),  # the last position would be 2^31
    (dict(B=1 << 16, S=1 << 15), seer.ERR_UNSUPPORTED),
    (dict(S=(1 << 27) + 1), seer.ERR_UNSUPPORTED),   # a launch holds less than 2^32 threads
    (dict(Hq=65535), seer.ERR_UNSUPPORTED),
    (dict(params=rope_params(freq=0)), seer.ERR_INVALID_ARG),
    (dict(params=rope_params(freq=FAKE + 4)), seer.ERR_INVALID_ARG),
    (dict(params=rope_params(rot=0)), seer.ERR_INVALID_ARG),
    (dict(params=rope_params(rot=144)), seer.ERR_INVALID_ARG),  # more than the head
    (dict(params=rope_params(rot=40)), seer.ERR_UNSUPPORTED),
    (dict(params=rope_params(inter=2)), seer.ERR_INVALID_ARG),
    (dict(params=rope_params(scale=math.nan)), seer.ERR_INVALID_ARG),
    (dict(params=rope_params(scale=math.inf)), seer.ERR_INVALID_ARG),
])
def test_rope_refuses(kw, status):
    assert rope_call(**kw) == status


def append_call(B=2, S=3, H=2, D=128, dtype=0, page=16, pages=8, rows=2, maxp=4, reserved=0, ks=None, kcs=None, ts=4,
                ps=3, params=rope_params(), k=FAKE, v=FAKE, kc=FAKE, vc=FAKE, table=FAKE, positions=FAKE, row_ids=None):
    st = ks or (H * S * D, S * D, D)
    cs = kcs or (H * page * D, page * D, D)
    d = decode._CACHE_DESC.pack(B, S, H, D, dtype, page, pages, rows, maxp, reserved, *st, *st, *cs, *cs, ts, ps)
    return seer.lib().seer_kv_append(d, params, k, v, kc, vc, table, positions, row_ids, None)


@pytest.mark.parametrize("kw,status", [
    *[({n: None}, seer.ERR_INVALID_ARG) for n in ("k", "v", "kc", "vc", "table", "positions")],
    *[({n: ODD}, seer.ERR_INVALID_ARG) for n in ("k", "v", "kc", "vc")],
    *[({n: FAKE + 1}, seer.ERR_INVALID_ARG) for n in ("table", "positions", "row_ids")],
    *[({n: 0}, seer.ERR_INVALID_ARG) for n in ("B", "S", "H", "page", "pages", "rows", "maxp")],
    (dict(reserved=1), seer.ERR_INVALID_ARG),
    (dict(D=80), seer.ERR_UNSUPPORTED),
    (dict(dtype=5), seer.ERR_INVALID_ARG),
    (dict(rows=1), seer.ERR_INVALID_ARG),            # two batch entries, one table row, no rows given
    (dict(ts=-4), seer.ERR_INVALID_ARG),
    (dict(ps=-1), seer.ERR_INVALID_ARG),
    (dict(ks=(100, 128, 128)), seer.ERR_UNSUPPORTED),
    (dict(kcs=(0, 2048, 128)), seer.ERR_INVALID_ARG),   # all pages at one place
    (dict(kcs=(4096, 2048, 64)), seer.ERR_INVALID_ARG),  # slots overlap
    (dict(page=1 << 16, maxp=1 << 15), seer.ERR_UNSUPPORTED),  # 2^31 tokens a row
    (dict(S=(1 << 26) + 1), seer.ERR_UNSUPPORTED),
    (dict(H=65536), seer.ERR_UNSUPPORTED),
    (dict(params=rope_params(rot=24)), seer.ERR_UNSUPPORTED),
])
def test_append_refuses(kw, status):
    assert append_call(**kw) == status


def paged_desc(B=2, Hq=8, Hkv=2, S=1, D=128, dtype=0, page=16, pages=8, maxp=4, reserved=0, qs=None, os_=None, cs=None,
               ts=4, ps=1):
    st = (Hq * S * D, S * D, D)
    cs = cs or (Hkv * page * D, page * D, D)
    return decode._CACHE_DESC.pack(B, Hq, Hkv, S, D, dtype, page, pages, maxp, reserved, *(qs or st), *(os_ or st), *cs,
                                   *cs, ts, ps)


def paged_call(params=None, scale=0.0, q=FAKE, kc=FAKE, vc=FAKE, table=FAKE, positions=FAKE, o=FAKE, lse=None, ws=FAKE,
               n=1 << 40, **kw):
    return seer.lib().seer_paged_attn(paged_desc(**kw), params, scale, q, kc, vc, table, positions, o, lse, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    *[({n: None}, seer.ERR_INVALID_ARG) for n in ("q", "kc", "vc", "table", "positions", "o")],
    *[({n: ODD}, seer.ERR_INVALID_ARG) for n in ("q", "kc", "vc", "o", "lse")],
    *[({n: 0}, seer.ERR_INVALID_ARG) for n in ("B", "Hq", "Hkv", "S", "page", "pages", "maxp")],
    (dict(Hkv=3), seer.ERR_INVALID_ARG),
    (dict(D=256), seer.ERR_UNSUPPORTED),
    (dict(dtype=-1), seer.ERR_INVALID_ARG),
    (dict(reserved=7), seer.ERR_INVALID_ARG),
    (dict(scale=math.nan), seer.ERR_INVALID_ARG),
    (dict(scale=math.inf), seer.ERR_INVALID_ARG),
    (dict(ws=None), seer.ERR_WORKSPACE),
    (dict(n=1000), seer.ERR_WORKSPACE),
    (dict(ws=FAKE + 16), seer.ERR_INVALID_ARG),
    (dict(qs=(4, 128, 128)), seer.ERR_UNSUPPORTED),
    (dict(os_=(1024, 0, 128)), seer.ERR_INVALID_ARG),
    (dict(cs=(4096, 2048, 12)), seer.ERR_UNSUPPORTED),
    (dict(ts=-1), seer.ERR_INVALID_ARG),
    (dict(ps=-1), seer.ERR_INVALID_ARG),
    (dict(page=1 << 20, maxp=1 << 11), seer.ERR_UNSUPPORTED),
    (dict(page=1 << 20, maxp=1 << 10, B=0), seer.ERR_INVALID_ARG),
    (dict(B=1 << 20, Hq=4096, Hkv=4096), seer.ERR_UNSUPPORTED),
    (dict(B=1 << 23), seer.ERR_UNSUPPORTED),         # 2^24 rows of 2 KV heads
    (dict(cs=(1 << 36, 2048, 128)), seer.ERR_UNSUPPORTED),
    (dict(params=rope_params(rot=8)), seer.ERR_UNSUPPORTED),
])
def test_paged_attention_refuses(kw, status):
    assert paged_call(**kw) == status


def test_paged_workspace_is_independent_of_the_lengths():
    L = seer.lib()
    need = L.seer_paged_attn_workspace_bytes(paged_desc())
    assert need > 0
    assert L.seer_paged_attn_workspace_bytes(paged_desc(maxp=1 << 14)) == need
    assert L.seer_paged_attn_workspace_bytes(paged_desc(D=32)) == 0
    assert L.seer_paged_attn_workspace_bytes(None) == 0
    assert paged_call(n=need - 1) == seer.ERR_WORKSPACE


def test_binding_refuses_host_tensors_and_wrong_types():
    q, k = torch.zeros(1, 4, 8, 128), torch.zeros(1, 2, 8, 128)
    f, scale = seer.rope_freqs(128, device="cpu")
    assert scale == 1.0
    with pytest.raises(ValueError):
        seer.rope(q, k, f)                             # no GPU tensors: nothing falls back to the CPU
    with pytest.raises(ValueError):
        seer.rope(q[0, 0], None, f)                    # two dimensions
    with pytest.raises(ValueError):
        seer.rope(q, k[:, :, :4], f)
    with pytest.raises(ValueError):
        seer.rope(q, None, None)
    with pytest.raises(ValueError):
        seer.rope(q, k, f, out=(q, None))
    kc = torch.zeros(4, 2, 16, 128)
    table, pos = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 8, dtype=torch.int32)
    with pytest.raises(ValueError):
        seer.kv_append(k, k, kc, kc, table, pos)
    with pytest.raises(ValueError):
        seer.kv_append(k, k[:, :1], kc, kc, table, pos)
    with pytest.raises(ValueError):
        seer.paged_attn(q, kc, kc, table, pos)


def test_frequencies():
    f, s = seer.rope_freqs(64, theta=500000.0, device="cpu")
    want = [500000.0 ** (-2 * p / 64) for p in range(32)]
    assert f.tolist() == want and s == 1.0
    lin, s = seer.rope_freqs(64, theta=500000.0, scaling="linear", factor=4.0, device="cpu")
    assert lin.tolist() == [x / 4 for x in want] and s == 1.0
    ntk, _ = seer.rope_freqs(64, theta=500000.0, scaling="ntk", factor=4.0, device="cpu")
    assert ntk[0] == 1.0 and ntk[-1].item() == pytest.approx(want[-1] / 4, rel=1e-12)
    bands, s = seer.rope_freqs(64, theta=500000.0, scaling="bands", factor=8.0, original_len=8192, device="cpu")
    assert s == 1.0
    for x, y in zip(want, bands.tolist()):
        turns = 8192 * x / (2 * math.pi)
        if turns >= 4:
            assert y == x
        elif turns <= 1:
            assert y == pytest.approx(x / 8, rel=1e-12)
        else:
            assert x / 8 < y < x
    yarn, s = seer.rope_freqs(64, scaling="yarn", factor=16.0, original_len=4096, device="cpu")
    assert s == pytest.approx(0.1 * math.log(16.0) + 1.0)
    assert yarn[0] == 1.0 and yarn[-1].item() == pytest.approx(10000.0 ** (-62 / 64) / 16, rel=1e-12)
    for bad in (dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=64, theta=0.0), dict(rot_dim=64, factor=0.5),
                dict(rot_dim=64, scaling="other"), dict(rot_dim=64, scaling="yarn", factor=2.0),
                dict(rot_dim=64, scaling="bands", original_len=64, low=4.0, high=4.0)):
        with pytest.raises(ValueError):
            seer.rope_freqs(**bad, device="cpu")


@pytest.mark.parametrize("start", [2 ** 31, -2 ** 31 - 1, 2 ** 32 + 5])
def test_binding_refuses_a_start_beyond_int32(start):
    q = torch.zeros(1, 2, 4, 64)
    with pytest.raises(ValueError, match="start"):
        seer.rope(q, None, seer.rope_freqs(64, device="cpu")[0], start=start)


def test_binding_refuses_keys_beside_no_queries():
    with pytest.raises(ValueError, match="heads"):
        seer.rope(torch.zeros(1, 0, 4, 64), torch.zeros(1, 2, 4, 64), seer.rope_freqs(64, device="cpu")[0])


def test_positions_are_axes_of_tokens():
    with pytest.raises(ValueError, match="positions"):
        decode._positions_of(torch.tensor(3, dtype=torch.int32), 1, 1, False)
