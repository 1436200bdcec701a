"""The loss of large finite logits, and of rows that are sure of their label.

The products of these tests are exact in fp32 (one channel counts, its factors have 8 or 11 bits), so what is
looked at is the softmax alone, however large its logits are."""
import numpy as np
import pytest

import sequence_util as U
import vocabulary_util as W

pytestmark = pytest.mark.gpu
U32 = W.U32


def softmax(z):
    """(p, z - largest, log of the sum of exp(z - largest)) in 64 bits, whatever the size of z: equal logits
    differ by 0."""
    d = z - z.max(axis=1, keepdims=True)
    e = np.exp(d)
    s = e.sum(axis=1, keepdims=True)
    return e / s, d, np.log(s[:, 0])


def p_error(p, d, dtype, v):
    """Of a probability: the difference to the largest logit, its product and log2(e) in it are rounded once
    each; the exponential and the sum of v of them, their quotient; what is kept of it between the products in 16 bits
    (vocabulary_util.bounds) and the operands' type.  Below 2^-126 fp32 has no more exponentials."""
    arg = 3 * U32 * np.minimum(-d, 100.0)
    return p * (2 * arg + (100 + v / 8192) * U32 + 2.0 ** -11 + U.HALF_ULP[dtype] * 1.01) + 2.0 ** -25


CASES = [  # rows, tokens, scale: 32 x 128, 128 x 128 and 256 x 256 tiles of logits
    (7, 700, 1.0), (40, 300, -0.375), (300, 12000, 0.75), (1100, 9000, -1.0), (1100, 9000, 3.0)]


@pytest.mark.parametrize("teacher", [False, True], ids=["labels", "teacher"])
@pytest.mark.parametrize("dtype,most", [("f16", 6e4), ("bf16", 2.0 ** 15), ("bf16", 2.0 ** 40)])
@pytest.mark.parametrize("rows,v,scale", CASES)
def test_large_logits(nnlib, rows, v, scale, dtype, most, teacher):
    """Logits from 1 to beyond 2^24, 2^31 and 2^80: many tokens share the largest of each row, and its probability."""
    rng = np.random.default_rng(rows + v)
    c = 8
    steps = U.round16(dtype)(np.sort(np.concatenate([-(most ** rng.random(12)), most ** rng.random(11)])))
    w, x = np.zeros((v, c)), np.zeros((rows, c))
    w[:, 0] = steps[rng.integers(0, len(steps), v)]
    x[:, 0] = U.round16(dtype)(rng.choice([-1.0, 1.0], rows) * most ** rng.random(rows))
    z = scale * np.outer(x[:, 0], w[:, 0])
    p, d, log_sum = softmax(z)
    # a half of the labels is among the most likely tokens
    best = np.array([rng.choice(np.flatnonzero(r == 0)) for r in d])
    label = np.where(rng.random(rows) < 0.5, best, rng.integers(0, v, rows))
    logits = np.zeros((rows, 1)) if teacher else None
    alpha = 2.0 ** -17 / most  # dx of fp16 stays finite
    got = W.loss_call(x, w, label[:, None], logits, dtype, scale, alpha=alpha, dw_dtype="f32")
    fwd = W.loss_call(x, w, label[:, None], logits, dtype, scale, train=False)
    at = d[np.arange(rows), label]
    loss, lse = log_sum - at, z.max(axis=1) + log_sum
    bound = (100 + v / 8192) * U32 + 4 * U32 * np.abs(at)
    for o in (got, fwd):
        assert np.all(np.abs(o["loss"].f64() - loss) <= bound)
        assert np.all(np.abs(o["lse"].f64() - lse) <= (100 + v / 8192) * U32 + 4 * U32 * np.abs(lse))
        assert np.all(o["loss"].f64() >= 0)
    dz, edz = p.copy(), p_error(p, d, dtype, v)
    dz[np.arange(rows), label] -= 1.0
    edz += U.HALF_ULP[dtype] * np.abs(dz)
    f = alpha * abs(scale)
    chain = (rows + v + 24) * 2 * U32
    dx, mag = f * np.sign(scale) * dz @ w, f * (edz + chain * np.abs(dz)) @ np.abs(w)
    U.close16(got["dx"].f64(), dx, dtype, mag * 1.01)
    dw, mag = f * np.sign(scale) * dz.T @ x, f * (edz + chain * np.abs(dz)).T @ np.abs(x)
    U.close32(got["dw"].f64(), dw, mag * 1.01 + 2.0 ** -140)


@pytest.mark.parametrize("teacher", [False, True], ids=["labels", "teacher"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 0.3, -0.7])
@pytest.mark.parametrize("size", [3.0, 30.0, 300.0, 1e4, 4e4])
@pytest.mark.parametrize("v", [90, 20000])
def test_certain_labels(nnlib, v, size, scale, dtype, teacher):
    """Where every other token lies more than 104 / log2(e) below the label, its probability is 1: the loss and all
    gradients are exactly 0, whatever the size of its logit."""
    rng = np.random.default_rng(int(size) + v)
    rows = c = 64
    x, w = np.zeros((rows, c)), np.zeros((v, c))
    label = rng.permutation(v)[:rows]
    at = np.arange(rows)
    sign = np.sign(scale)
    x[at, at] = 1.0 + rng.random(rows)
    w[:] = -600.0 * sign
    w[label] = -600.0 * sign
    w[label, at] = size * (1.0 + 0.6 * rng.random(rows)) * sign
    x, w = U.round16(dtype)(x), U.round16(dtype)(w)
    logits = np.ones((rows, 1)) if teacher else None
    got = W.loss_call(x, w, label[:, None], logits, dtype, scale, dw_dtype="f32", grad_scale=1024.0)
    z = np.float32(scale).astype(np.float64) * x[at, at] * w[label, at]
    assert np.all(np.abs(got["lse"].f64() - z) <= 4 * U32 * np.abs(z))
    for key in ("loss", "dx", "dw"):
        assert not got[key].f64().any(), key
    fwd = W.loss_call(x, w, label[:, None], logits, dtype, scale, train=False)
    assert not fwd["loss"].f64().any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("teacher", [False, True], ids=["labels", "teacher"])
def test_the_loss_is_never_negative(nnlib, dtype, teacher):
    """Rows that are more or less sure, with products that are rounded."""
    rng = np.random.default_rng(21)
    rows, c, v = 300, 200, 1000
    w = U.normal(rng, (v, c), dtype, 1.0)
    label = rng.integers(0, v, rows)
    x = U.round16(dtype)(w[label] * (10.0 ** rng.uniform(-2.5, 1.5, (rows, 1))))
    logits = np.ones((rows, 1)) if teacher else None
    loss = W.loss_call(x, w, label[:, None], logits, dtype)["loss"].f64()
    assert np.all(loss >= 0)
    if not teacher:  # its targets have sums of their own
        assert loss.min() == 0
