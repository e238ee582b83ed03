"""Both sides of the limits that include/seer_decode.h names (no GPU needed: every call here returns from
argument validation, which touches no device)."""
import os

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")
if not os.path.exists(seer.LIB_PATH):
    pytest.skip("libseer.so not built", allow_module_level=True)

from test_decode_abi import paged_call  # noqa: E402


def test_scale_whose_product_with_log2_e_is_infinite():
    """2^127 log2(e) is 2.45e38, FLT_MAX log2(e) beyond fp32.  (Without a workspace no call is made: that is refused after
    the scale.)"""
    for scale in (2.0 ** 127, 0.0, -2.0 ** 127, -3.4028234e38):
        assert paged_call(scale=scale, ws=None) == seer.ERR_WORKSPACE
    for scale in (2.0 ** 127 * (1 + 2.0 ** -23), 2.4e38, 3.4028234e38):
        assert paged_call(scale=scale, ws=None) == seer.ERR_INVALID_ARG
