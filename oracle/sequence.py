"""fp64 oracle of the gated sequence block's operators, from their definitions
(include/nnconv.h): root-mean-square norm with the residual's addition, gated
linear recurrence, AdamW with fp32 or 8-bit moments.

Test infrastructure only: plain numpy, token by token and step by step, no
code in common with the HIP library.  Operands are float64 arrays that hold
the exact values of the 16-bit inputs; results are not rounded, apart from the
norm's stored residual stream (`round16`, the caller's rounding to the storage
type) and the moments' 8-bit codes.
"""
from __future__ import annotations

import numpy as np

GATE_LIMIT = 80.0
F8_LARGEST = {"m": 448.0, "v": 57344.0}   # e4m3, e5m2
BLOCK = 64


# --- norm ---------------------------------------------------------------------

def rmsnorm_fwd(x, residual, gain, eps, round16):
    """(r, rstd, y) of [rows][c] float64 arrays."""
    r = x if residual is None else round16(x + residual)
    rstd = 1.0 / np.sqrt((r * r).mean(axis=1) + eps)
    return r, rstd, r * rstd[:, None] * gain


def rmsnorm_bwd(r, rstd, gain, dy, dsum=None):
    """(dx, dgain) before the loss-scale step."""
    xh = r * rstd[:, None]
    p = dy * gain
    dx = rstd[:, None] * (p - xh * (p * xh).mean(axis=1, keepdims=True))
    if dsum is not None:
        dx = dx + dsum
    return dx, (dy * xh).sum(axis=0)


def quantise_scales(y, group):
    """max |y| / 448 per row (group 0) or group of channels; NaNs are passed over."""
    rows, c = y.shape
    group = group or c
    mag = np.where(np.isnan(y), 0.0, np.abs(y))
    s = np.stack([mag[:, i:i + group].max(axis=1) for i in range(0, c, group)], axis=1) / 448.0
    return np.where(s < 2.0 ** -126, 0.0, s)


# --- recurrence ---------------------------------------------------------------

def gates(f, bias):
    z = f + (0.0 if bias is None else bias)
    z = np.where(np.isnan(z), z, np.clip(z, -GATE_LIMIT, GATE_LIMIT))
    return 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))


def _lengths(lengths, n, t):
    return [t] * n if lengths is None else [min(max(int(v), 0), t) for v in lengths]


def recurrence_fwd(x, f, bias, g=None, lengths=None, h0=None):
    """(y, h) of [n][t][c]: h[i][j] is the state before token j, h[i][t] the last."""
    n, t, c = x.shape
    a, b = gates(f, bias)
    h = np.zeros((n, t + 1, c))
    if h0 is not None:
        h[:, 0] = h0
    y = np.zeros((n, t, c))
    for i, length in enumerate(_lengths(lengths, n, t)):
        for j in range(t):
            if j >= length:
                h[i, j + 1] = h[i, j]
                continue
            h[i, j + 1] = a[i, j] * h[i, j] + b[i, j] * x[i, j]
            y[i, j] = h[i, j + 1] if g is None else h[i, j + 1] * g[i, j] / (1.0 + np.exp(-g[i, j]))
    return y, h


def recurrence_bwd(x, f, bias, dy, h, g=None, lengths=None, dht=None):
    """(dx, df, dg, dh0, dbias) before the loss-scale step; h as recurrence_fwd gives it."""
    n, t, c = x.shape
    a, b = gates(f, bias)
    dx, df, dg = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    dh0 = np.zeros((n, c)) if dht is None else np.array(dht, dtype=np.float64)
    for i, length in enumerate(_lengths(lengths, n, t)):
        for j in range(length - 1, -1, -1):
            own = dy[i, j]
            if g is not None:
                s = 1.0 / (1.0 + np.exp(-g[i, j]))
                dg[i, j] = own * h[i, j + 1] * (s + g[i, j] * s * (1.0 - s))
                own = own * g[i, j] * s
            d = dh0[i] + own
            dx[i, j] = d * b[i, j]
            df[i, j] = d * (h[i, j] - x[i, j]) * a[i, j] * b[i, j]
            dh0[i] = d * a[i, j]
    return dx, df, (None if g is None else dg), dh0, df.sum(axis=(0, 1))


# --- AdamW --------------------------------------------------------------------

def adamw_moments(m, v, grad, scale, beta1, beta2):
    g = grad / scale
    return beta1 * m + (1.0 - beta1) * g, beta2 * v + (1.0 - beta2) * g * g


def adamw_master(master, m, v, step, lr, beta1, beta2, eps, decay):
    """The master after step `step` (1 for the first), from the new moments."""
    mh = m / (1.0 - beta1 ** step)
    vh = v / (1.0 - beta2 ** step)
    return master - lr * (mh / (np.sqrt(vh) + eps) + decay * master)


def dither(seed, step, tensor, count):
    """(for m, for v): numbers in (0, 1) that say where each element is rounded."""
    mask = 0xFFFFFFFF
    key = (tensor * 0x6C8E9CF5 + step * 0xB5297A4D + seed * 0x68E31DA4) & mask
    i = np.arange(count, dtype=np.uint64)
    h = (i * np.uint64(0x9E3779B1) + np.uint64(key)) & np.uint64(mask)
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x2C1B3C6D)) & np.uint64(mask)
    h = ((h ^ (h >> np.uint64(15))) * np.uint64(0x297A2D39)) & np.uint64(mask)
    h = h ^ (h >> np.uint64(16))
    return tuple(((p & np.uint64(0xFFFF)).astype(np.float64) + 0.5) / 65536.0 for p in (h, h >> np.uint64(16)))


def encode(x, u, which):
    """(values the codes stand for, scales): values on the 8-bit grid nearest below or above x by u."""
    top, low, bits = (8, -6, 3) if which == "m" else (15, -14, 2)
    out = np.zeros(x.shape)
    scales = np.zeros(-(-x.size // BLOCK))
    for b in range(scales.size):
        part = slice(b * BLOCK, min((b + 1) * BLOCK, x.size))
        v = x[part]
        fine = np.isfinite(v)
        most = np.abs(v[fine]).max(initial=0.0)
        k = -127
        if most > 0.0:
            k = max(-127, int(np.floor(np.log2(most))) - top)
            while most > F8_LARGEST[which] * 2.0 ** k:
                k += 1
            while k > -127 and most <= F8_LARGEST[which] * 2.0 ** (k - 1):
                k -= 1
        scales[b] = 2.0 ** k
        y = np.where(fine, np.abs(v), 0.0) / 2.0 ** k
        e = np.maximum(np.floor(np.log2(np.where(y > 0.0, y, 1.0))), low)
        ulp = 2.0 ** (e - bits)
        r = np.floor(y / ulp + u[part])
        if which == "v":
            r = np.where((r == 0.0) & (y > 0.0), 1.0, r)
        r = np.minimum(r * ulp, F8_LARGEST[which])
        out[part] = np.where(fine, np.copysign(r, v) * 2.0 ** k, np.nan)
    return out, scales
