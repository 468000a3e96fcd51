"""moe_add_rmsnorm's codes are e4m3(y / s) by an fp32 division, for every fp32 y.  A row of ones with eps = 0 has 1/rms = 1, so y is the gain as it is."""
import numpy as np
import pytest
import torch

from oracle import fp_formats as ff
from training_common import Context

pytestmark = pytest.mark.gpu


def _codes(moe, gain, rows):
    cols = gain.size
    x = torch.ones((rows, cols), device="cuda")
    q, s = torch.empty((rows, cols), dtype=torch.uint8, device="cuda"), torch.empty((cols // 128, rows), device="cuda")
    with Context(moe, reserve=False) as ctx:
        moe.moe_add_rmsnorm(ctx, x, None, torch.from_numpy(gain).cuda(), 0.0, q=q, scales=s)
        torch.cuda.synchronize()
    return q.cpu().numpy(), s.cpu().numpy()


def _check(moe, gain, rows=1):
    q, s = _codes(moe, gain, rows)
    g = gain.reshape(-1, 128)
    amax = np.abs(g).max(axis=1)
    scale = np.where(amax == 0, np.float32(1), amax / np.float32(448))
    assert scale.dtype == np.float32
    want = ff.e4m3_encode((g / scale[:, None]).astype(np.float64)).reshape(-1)
    for r in range(rows):
        assert np.array_equal(s[:, r], scale)
        assert np.array_equal(q[r], want), np.flatnonzero(q[r] != want)


@pytest.mark.parametrize("rows", [1, 4000])
@pytest.mark.parametrize("std", [1.0, 1e-24, 1e24, 1e-38])
def test_random_values(gpu_lib, std, rows):
    rng = np.random.default_rng([rows, int(abs(np.log10(std)))])
    n = 32768 if rows == 1 else 4096
    gain = (rng.normal(size=n) * 2.0 ** rng.uniform(-20, 0, n) * std).astype(np.float32)
    gain[128:256] = 0
    _check(gpu_lib, gain, rows)


def test_scales_of_nothing_but_ones(gpu_lib):
    """Powers of two over a scale of (2 - 2^-23) 2^k: a quotient a little above a tie"""
    groups = []
    for k in range(-60, 61, 2):
        amax = np.nextafter(np.float32(1.75), np.float32(0)) * np.float32(2.0) ** k
        scale = np.float32(amax) / np.float32(448)
        assert scale.view(np.uint32) & 0x7FFFFF == 0x7FFFFF
        g = np.float32(2.0) ** (k - np.arange(128) % 24).astype(np.float32)
        g[0], g[1::2] = amax, -g[1::2]
        groups.append(g.astype(np.float32))
    _check(gpu_lib, np.concatenate(groups))


def test_maxima_whose_scale_underflows(gpu_lib):
    """amax / 448 is zero in fp32 up to 448 * 2^-150: scale 1 and codes of zero, with zeros in the group and without"""
    gain = np.zeros(512, np.float32)
    gain[:3] = 1e-43, -1e-44, 1.5e-45
    gain[128:256] = 1e-44
    gain[256:384] = np.float32(2.0) ** -140                    # (the scale is the smallest subnormal)
    gain[384] = 1.0
    q, s = _codes(gpu_lib, gain, 3)
    assert (s[:2] == 1).all() and (s[2] == np.float32(2.0) ** -149).all() and (s[3] == np.float32(1) / np.float32(448)).all()
    assert (q[:, :256] & 0x7F == 0).all() and (q[:, 385:] & 0x7F == 0).all() and (q[:, 384] == 0x7E).all()
    assert (q[:, 256:384] == 0x7E).all()                       # 2^-140 / 2^-149 = 512, the largest code
