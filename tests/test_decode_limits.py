"""Both sides of the limits that include/seer_decode.h names (no GPU needed: every call here returns from
argument validation, which touches no device)."""
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

from test_decode_abi import paged_call, paged_desc  # noqa: E402


def test_scale_whose_product_with_log2_e_is_infinite():
    """2^127 log2(e) is 2.45e38, FLT_MAX log2(e) beyond fp32.  (Without a workspace no call is made: that is refused after
    the scale.)"""
    for scale in (2.0 ** 127, 0.0, -2.0 ** 127, -3.4028234e38):
        assert paged_call(scale=scale, ws=None) == seer.ERR_WORKSPACE
    for scale in (2.0 ** 127 * (1 + 2.0 ** -23), 2.4e38, 3.4028234e38):
        assert paged_call(scale=scale, ws=None) == seer.ERR_INVALID_ARG


@pytest.mark.parametrize("kw,fits", [
    (dict(B=1 << 20, Hq=8 * 16, Hkv=8), True),                  # 2^23 KV heads of a block of 16 rows each
    (dict(B=(1 << 20) + 1, Hq=8 * 16, Hkv=8), False),
    (dict(B=1 << 20, Hq=8, Hkv=8), True),                       # ... of one row each
    (dict(B=1 << 20, Hq=8 * 17, Hkv=8), False),                 # 17 rows are two blocks
    (dict(B=1 << 19, Hq=8 * 17, Hkv=8), True),
    (dict(B=1 << 16, Hq=8, Hkv=8, S=256), True),                # 2^19 KV heads of 16 blocks
    (dict(B=1 << 16, Hq=8, Hkv=8, S=257), False),
    (dict(B=5 << 20, Hq=16, Hkv=1), True),
    (dict(B=1, Hq=1, Hkv=1, S=1 << 23), True),                  # 2^23 rows of one KV head
    (dict(B=1, Hq=1, Hkv=1, S=(1 << 23) + 1), False),
    (dict(B=16, Hq=2, Hkv=1, S=1 << 22), True),
    (dict(B=17, Hq=2, Hkv=1, S=1 << 22), False),
    (dict(B=2 ** 31 - 1, Hq=2 ** 31 - 1, Hkv=2 ** 31 - 1, S=2 ** 31 - 1), False),
    (dict(B=2 ** 31 - 1, Hq=2 ** 31 - 1, Hkv=1, S=2 ** 31 - 1), False),
])
def test_query_rows_and_their_blocks(kw, fits):
    st = (128, 128, 128)  # (strides take no part in the count)
    need = seer.lib().seer_paged_attn_workspace_bytes(paged_desc(**kw, qs=st, os_=st))
    assert (need > 0) == fits
    assert paged_call(**kw, qs=st, os_=st, ws=None) == (seer.ERR_WORKSPACE if fits else seer.ERR_UNSUPPORTED)
