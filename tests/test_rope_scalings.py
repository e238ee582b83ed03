"""The long-context frequencies of rope_freqs plane by plane against their formulas, and a rotation by them."""
import math

import pytest

torch = pytest.importorskip("torch")
seer = pytest.importorskip("paper_2410_13276_amd")

from decode_ref import assert_rounded, rotate  # noqa: E402


@pytest.mark.parametrize("rot,theta,length,factor", [(128, 500000.0, 8192, 8.0), (64, 10000.0, 4096, 16.0)])
def test_every_plane_of_the_ramps(rot, theta, length, factor):
    """The share that a plane keeps is linear in its turns over the trained length, between 1 and 32 turns (arXiv 2309.00071,
    by parts) or 1 and 4.  Powers, products and the sum in 64 bits: within 16 steps of 2^-53."""
    for scaling, high, scale in (("yarn", 32.0, 0.1 * math.log(factor) + 1.0), ("bands", 4.0, 1.0)):
        f, s = seer.rope_freqs(rot, theta=theta, scaling=scaling, factor=factor, original_len=length, device="cpu")
        assert s == pytest.approx(scale, rel=1e-15)
        between = 0
        for p, got in enumerate(f.tolist()):
            plain = theta ** (-2.0 * p / rot)
            turns = length * plain / (2 * math.pi)
            keep = 1.0 if turns > high else 0.0 if turns < 1.0 else (turns - 1.0) / (high - 1.0)
            between += 0.0 < keep < 1.0
            assert got == pytest.approx((1.0 - keep) * plain / factor + keep * plain, rel=16 * 2.0 ** -53)
        assert between >= 2


@pytest.mark.gpu
@pytest.mark.parametrize("scaling", ["linear", "ntk", "bands", "yarn"])
def test_rotation_by_scaled_frequencies(scaling):
    gen = torch.Generator().manual_seed(13)
    f, scale = seer.rope_freqs(128, theta=500000.0, scaling=scaling, factor=8.0, original_len=8192)
    x = torch.randn(1, 2, 40, 128, generator=gen)
    pos = torch.randint(0, 65536, (40,), generator=gen, dtype=torch.int32)
    y, _ = seer.rope(x.cuda(), None, f, pos.cuda(), rope_scale=scale)
    ref, err = rotate(x, pos[None, None, :], f.cpu(), scale)
    assert_rounded(y.cpu(), ref, err)
