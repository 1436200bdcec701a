"""Infinities and NaNs through the sequence block's operators: each in its place and with its sign, as the definition
has them, and the values beside them within the bounds that the operators' own tests derive."""
import numpy as np
import pytest

from oracle import sequence as S

import sequence_util as U
import strict_util as X
import test_gpu_rmsnorm as N
from test_gpu_recurrence import ULP, Case

pytestmark = pytest.mark.gpu
INF = np.inf


@pytest.mark.parametrize("c", [5, 8, 100, 771, 2048, 9000, 20000])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_norm_rows(nnlib, c, dtype):
    x, res, gain, _ = N.inputs(16, c, dtype, True)
    top = float(U.torch().finfo(U.tdtype(dtype)).max)
    x[1, c // 2], x[2, 0], x[3, c - 1] = INF, -INF, np.nan
    res[4, 1], x[4, 1] = INF, -INF       # their sum is NaN
    res[5, 2] = -INF
    x[6], res[6] = top, top              # the sum passes the type's range, up
    x[7], res[7] = -top, -top            # and down
    gain[0], gain[1] = 3e6, -3e6         # y passes fp16's range with either sign
    gain = gain.astype(np.float32).astype(np.float64)
    with np.errstate(all="ignore"):
        r, rstd, y = S.rmsnorm_fwd(x, res, gain, N.EPS, U.round16(dtype))
    b = N.forward(16, c, dtype, x, res, gain, "own", 0)
    X.close16(b["S"].f64(), r, dtype, 0.0)
    # a row whose mean square passes fp32's range has rstd 0
    rstd = np.where((r * r).mean(axis=1) > np.finfo(np.float32).max, 0.0, rstd)
    with np.errstate(all="ignore"):
        y = r * rstd[:, None] * gain
    X.close32(b["rstd"].f64(), rstd, N.slack(c) * X.finite(rstd))
    X.close16(b["Y"].f64(), y, dtype, N.slack(c) * X.finite(y))


def bounds(c, h, a, b, dy, dht):
    """Magnitudes as in the recurrence's own tests, from what is finite."""
    z = X.finite(c.f + (0 if c.bias is None else c.bias)).max()
    steps = min(c.t, float((1.0 / X.finite(np.where(b > 0, b, 1.0)).clip(1e-40)).max()))
    big = np.maximum(X.finite(h).max(axis=1), X.finite(c.x).max(axis=1))[:, None]
    sil = 1.0 if c.g is None else np.abs(c.g) / (1.0 + np.exp(-c.g))
    dmag, carry = np.zeros_like(c.x), X.finite(dht)
    for j in range(c.t - 1, -1, -1):
        dmag[:, j] = carry + X.finite(dy[:, j]) * (sil if c.g is None else sil[:, j])
        carry = dmag[:, j] * X.finite(a[:, j])
    return z, steps, big, sil, dmag.max(axis=1)[:, None]


@pytest.mark.parametrize("t", [1, 5, 40, 150, 1100])
@pytest.mark.parametrize("c", [1, 20, 40, 64, 90, 131])
@pytest.mark.parametrize("with_g", [True, False])
def test_recurrence(nnlib, t, c, with_g):
    """Infinite and NaN values and gates; the gradients of a finite forward pass with infinite and NaN dy and dht."""
    case = Case(4, t, c, "bf16", with_g=with_g, seed=41)
    j = t // 3
    case.x[0, j, 0], case.x[1, j, c // 2], case.x[2, j, c - 1] = INF, -INF, np.nan
    case.f[3, j, 0] = np.nan
    if c > 8:
        case.f[0, t // 2, 3], case.f[0, t // 2, 4] = INF, -INF
        case.x[3, 0, 5], case.x[3, t - 1, 5] = INF, -INF  # one after the other: NaN, or the second where there is one token
        case.h0[1, 6], case.h0[2, 6], case.h0[3, 7] = INF, -INF, np.nan
        if with_g:
            case.g[0, j, 0], case.g[1, t - 1, 7] = -3.0, np.nan
    y, ht = case.forward()
    with np.errstate(all="ignore"):
        ry, h = S.recurrence_fwd(case.x, case.f, case.bias, case.g, None, case.h0)
        a, b = S.gates(case.f, case.bias)
    z, steps, big, sil, _ = bounds(case, h, a, b, case.dy, case.dht)
    k = ULP * (max(z, 80.0) + 8 + 2 * steps)
    X.close16(y, ry, "bf16", k * big * X.finite(sil) + 8 * ULP * X.finite(ry))
    X.close32(ht, h[:, -1], k * big[:, 0])


@pytest.mark.parametrize("t", [1, 5, 40, 150, 1100])
@pytest.mark.parametrize("c", [1, 20, 40, 64, 90, 131])
@pytest.mark.parametrize("with_g", [True, False])
def test_recurrence_gradients(nnlib, t, c, with_g):
    case = Case(4, t, c, "bf16", with_g=with_g, seed=42)
    j = t // 2
    case.dy[0, j, 0], case.dy[1, j, c // 2], case.dy[2, j, c - 1] = INF, -INF, np.nan
    case.dht[3, 0] = -INF
    if c > 8:
        case.dht[1, 3], case.dht[2, 3] = INF, np.nan
    case.forward()
    got = case.backward()
    with np.errstate(all="ignore"):
        _, h = S.recurrence_fwd(case.x, case.f, case.bias, case.g, None, case.h0)
        a, b = S.gates(case.f, case.bias)
        ref = S.recurrence_bwd(case.x, case.f, case.bias, case.dy, h, case.g, None, case.dht)
    z, steps, big, sil, dbig = bounds(case, h, a, b, case.dy, case.dht)
    k4 = ULP * (z + 16 + 4 * steps)
    X.close16(got[0], ref[0], "bf16", k4 * dbig * b)
    X.close16(got[1], ref[1], "bf16", k4 * dbig * 4 * big * a * b)
    if with_g:
        X.close16(got[2], ref[2], "bf16", k4 * 2 * X.finite(case.dy) * big * (1 + np.abs(case.g)))
    X.close32(got[3], ref[3], k4 * np.maximum(dbig[:, 0], X.finite(case.dht)))
    # sums over an infinite column are infinite or NaN, the others finite, and the flag is set for them
    bad = ~np.isfinite(ref[1]).all(axis=(0, 1))
    assert np.array_equal(~np.isfinite(got[4]), bad) and got[5] == int(bad.any())


@pytest.mark.parametrize("t", [1, 150])
def test_recurrence_past_the_types_range(nnlib, t):
    """y and dx past fp16's largest value become infinities of their sign."""
    case = Case(2, t, 40, "f16", seed=43)
    case.x[:, :, :8], case.x[:, :, 8:16] = 60000.0, -60000.0
    case.h0[:, :8], case.h0[:, 8:16] = 60000.0, -60000.0
    case.g[:, :, :16:2], case.g[:, :, 1:16:2] = 5.0, 9.0
    y, ht = case.forward()
    ry, h = S.recurrence_fwd(case.x, case.f, case.bias, case.g, None, case.h0)
    assert np.isinf(y).any() and np.abs(ry).max() > 65520
    z, steps, big, sil, _ = bounds(case, h, *S.gates(case.f, case.bias), case.dy, case.dht)
    k = ULP * (z + 8 + 2 * steps)
    X.close16(y, ry, "f16", k * big * sil + 8 * ULP * np.abs(ry))
    X.close32(ht, h[:, -1], k * big[:, 0])
