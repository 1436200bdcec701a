"""The 8-bit norm's scales and codes, bit by bit: scale = max|y| / 448 and q = e4m3(y / scale) with
both quotients rounded to fp32 as a division is.

Rows of 1 and -1 with eps = 0 have rstd = 1 exactly, so that |y| is the gain, whatever number that
is: there is no arithmetic in front of the quotients and no tolerance on them."""
import numpy as np
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

pytestmark = pytest.mark.gpu
f32 = np.float32


def gains(rng, c, group, exponent):
    """Gains whose quotients lie on, just below and just above the ties between two codes."""
    g = np.empty(c, f32)
    for lo in range(0, c, group):
        part = g[lo:lo + group]
        part[0] = f32(np.ldexp(1.0 + rng.random(), exponent + int(rng.integers(-3, 4))))
        scale = part[0] / f32(448)
        tie = ((rng.integers(8, 15, part.size - 1) + 0.5) * 2.0 ** rng.integers(-9, 5, part.size - 1)).astype(f32)
        at = (tie * scale).astype(f32)
        for _ in range(2):
            at = np.where(rng.random(at.size) < 0.3, np.nextafter(at, f32(0)), np.where(rng.random(at.size) < 0.3, np.nextafter(at, f32(np.inf)), at))
        part[1:] = np.minimum(at, part[0])
    return g * rng.choice(np.array([1, -1], f32), c)


# every layout of threads, rows whose last vector is shared, and the kernels of very short and very long rows
@pytest.mark.parametrize("c", [4, 8, 16, 32, 64, 100, 128, 256, 512, 771, 1001, 1024, 2048, 4096, 4100, 8192, 16384, 20000])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("exponent", [0, -112, 100])
def test_scales_and_codes_are_the_quotients(nnlib, c, group, exponent):
    t = U.torch()
    rng = np.random.default_rng(c + group)
    rows, wide = 5, group or c
    g = gains(rng, c, wide, exponent)
    sign = rng.choice([1.0, -1.0], (rows, c))
    X, G = U.Buf(sign, "f16"), U.Buf(g, "f32")
    Q, S, R = U.Buf(dtype="e4m3", shape=(rows, c)), U.Buf(dtype="f32", shape=(rows, -(-c // wide))), U.Buf(dtype="f32", shape=(rows,))
    d = nc.nnconv_rmsnorm_desc(rows, c, U.CODE["f16"], group, 0.0)
    nc.check(nc.nnconv_rmsnorm_fwd_q8(d, X.data_ptr(), None, G.data_ptr(), None, Q.data_ptr(), S.data_ptr(), R.data_ptr(), None))
    assert np.all(R.f64() == 1.0)
    y = sign.astype(f32) * g
    most = np.stack([np.abs(y[:, lo:lo + wide]).max(axis=1) for lo in range(0, c, wide)], axis=1)
    scale = most / f32(448)
    assert np.all(scale >= 2.0 ** -126)
    assert np.array_equal(S.host().numpy(), scale)
    want = t.from_numpy(y / np.repeat(scale, wide, axis=1)[:, :c]).to(t.float8_e4m3fn)
    assert np.array_equal(Q.host().view(t.uint8).numpy(), want.view(t.uint8).numpy())
