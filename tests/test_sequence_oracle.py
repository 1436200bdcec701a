"""Pins of the sequence operators' oracle: gradients against differences of the
forward functions, closed forms, the 8-bit grid against torch's types."""
import numpy as np
import pytest

from oracle import sequence as S

EPS = 1e-6


def differences(f, x, h=1e-6):
    """d f / d x by central differences, f a number."""
    out = np.zeros_like(x)
    flat, o = x.reshape(-1), out.reshape(-1)
    for i in range(flat.size):
        old = flat[i]
        flat[i] = old + h
        up = f()
        flat[i] = old - h
        down = f()
        flat[i] = old
        o[i] = (up - down) / (2 * h)
    return out


@pytest.mark.parametrize("c", [1, 2, 7])
def test_norm_gradient(c):
    rng = np.random.default_rng(c)
    r, gain = rng.standard_normal((3, c)), rng.standard_normal(c)
    dy, dsum = rng.standard_normal((3, c)), rng.standard_normal((3, c))
    _, rstd, _ = S.rmsnorm_fwd(r, None, gain, EPS, None)
    dx, dgain = S.rmsnorm_bwd(r, rstd, gain, dy, dsum)

    def loss():
        return float((S.rmsnorm_fwd(r, None, gain, EPS, None)[2] * dy).sum() + (r * dsum).sum())
    assert np.allclose(differences(loss, r), dx, rtol=1e-6, atol=1e-6)
    assert np.allclose(differences(loss, gain), dgain, rtol=1e-6, atol=1e-6)


def test_norm_closed_forms():
    # a row of one value v: y = sign(v) gain without eps
    _, rstd, y = S.rmsnorm_fwd(np.full((1, 5), -3.0), None, np.arange(5.0), 0.0, None)
    assert np.allclose(y, -np.arange(5.0)) and np.allclose(rstd, 1.0 / 3.0)
    # orthogonal to the row at gain 1: the gradient of y at r has no part along r (eps = 0)
    rng = np.random.default_rng(0)
    r, dy = rng.standard_normal((2, 9)), rng.standard_normal((2, 9))
    _, rstd, _ = S.rmsnorm_fwd(r, None, np.ones(9), 0.0, None)
    assert np.allclose((S.rmsnorm_bwd(r, rstd, np.ones(9), dy)[0] * r).sum(axis=1), 0.0, atol=1e-12)


@pytest.mark.parametrize("with_g", [False, True])
@pytest.mark.parametrize("t,lengths", [(1, None), (5, None), (6, [0, 1, 4]), (4, [-2, 9, 4])])
def test_recurrence_gradient(t, lengths, with_g):
    rng = np.random.default_rng(t)
    n, c = 3, 2
    x, f, g = (rng.standard_normal((n, t, c)) for _ in range(3))
    bias, h0 = rng.standard_normal(c), rng.standard_normal((n, c))
    dy, dht = rng.standard_normal((n, t, c)), rng.standard_normal((n, c))
    gg = g if with_g else None
    _, h = S.recurrence_fwd(x, f, bias, gg, lengths, h0)
    dx, df, dg, dh0, dbias = S.recurrence_bwd(x, f, bias, dy, h, gg, lengths, dht)

    def loss():
        y, hh = S.recurrence_fwd(x, f, bias, gg, lengths, h0)
        return float((y * dy).sum() + (hh[:, -1] * dht).sum())
    pairs = [(x, dx), (f, df), (bias, dbias), (h0, dh0)] + ([(g, dg)] if with_g else [])
    for v, d in pairs:
        assert np.allclose(differences(loss, v), d, rtol=1e-6, atol=1e-7)


def test_recurrence_closed_forms():
    # gates at one half, x = 1: h_t = 1 - 2^-t; an open gate keeps the state, a shut one takes x
    x = np.ones((1, 6, 1))
    y, h = S.recurrence_fwd(x, np.zeros_like(x), None)
    assert np.allclose(y[0, :, 0], 1.0 - 0.5 ** np.arange(1, 7))
    y, _ = S.recurrence_fwd(x, np.full_like(x, 1e4), None, h0=np.full((1, 1), 7.0))
    assert np.allclose(y, 7.0)
    y, _ = S.recurrence_fwd(x, np.full_like(x, -1e4), None, h0=np.full((1, 1), 7.0))
    assert np.allclose(y, 1.0)


def test_adamw_first_step_is_a_signed_step():
    # from zero moments the first step is lr * g / |g| whatever the betas
    g = np.array([3.0, -0.5, 1e-3])
    m, v = S.adamw_moments(np.zeros(3), np.zeros(3), g * 8.0, 8.0, 0.9, 0.999)
    w = S.adamw_master(np.ones(3), m, v, 1, 0.1, 0.9, 0.999, 0.0, 0.0)
    assert np.allclose(w, 1.0 - 0.1 * np.sign(g))
    # decay alone
    w = S.adamw_master(np.ones(3), np.zeros(3), np.zeros(3), 1, 0.1, 0.9, 0.999, 1e-8, 0.5)
    assert np.allclose(w, 0.95)


@pytest.mark.parametrize("which,kind", [("m", "float8_e4m3fn"), ("v", "float8_e5m2")])
def test_codes_lie_on_the_types_grid(which, kind):
    import torch
    rng = np.random.default_rng(3)
    x = rng.standard_normal(640) * np.exp(rng.standard_normal(640) * 4)
    x = np.abs(x) if which == "v" else x
    x[64:128] = 0.0
    vals, scales = S.encode(x, rng.random(640), which)
    codes = vals / np.repeat(scales, 64)
    back = torch.from_numpy(codes).to(getattr(torch, kind)).double().numpy()
    assert np.array_equal(back, codes)
    assert scales[1] == 2.0 ** -127 and not vals[64:128].any()
    top = S.F8_LARGEST[which]
    for b in (0, 2, 9):
        most = np.abs(x[64 * b:64 * b + 64]).max()
        assert top / 2 * scales[b] < most <= top * scales[b]
    if which == "v":
        assert np.all(vals[x > 0] > 0)


def test_rounding_keeps_the_average():
    x = np.tile(np.array([1.0, 0.31, 0.077, 1e-3, 0.9003]), 64 * 200)[:64 * 1000]
    got = np.zeros(5)
    for step in range(20):
        u, _ = S.dither(5, step, 0, x.size)
        vals, _ = S.encode(x, u, "m")
        got += np.array([vals[i::5].mean() for i in range(5)]) / 20
    # 20 * 12800 draws of a rounding whose spacing is at most 1/8 of the value:
    # the mean's deviation is at most value / 16 / 506, five of them allowed
    assert np.all(np.abs(got - x[:5]) <= 5 * np.maximum(x[:5], 2.0 ** -15) / 16 / 506)
