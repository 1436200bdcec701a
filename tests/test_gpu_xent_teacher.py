"""A teacher's logits at the ends of their range, as its masks have them, with factors of either sign."""
import numpy as np
import pytest

from oracle import vocabulary as V

import sequence_util as U
import vocabulary_util as W

pytestmark = pytest.mark.gpu
U32 = W.U32
LOWEST = {"f32": -float(np.finfo(np.float32).max), "f16": -65504.0, "bf16": -float(255 * 2.0 ** 120)}


def check(got, x, w, targets, teacher, dtype, scale):
    """As vocabulary_util.check_loss, whose bounds grow with the largest of a teacher's logits: those of an entry whose share is
    0 do not count here, and the others are compared with the row's largest.  A row whose logits are no numbers is
    one whose loss and gradient are none either."""
    with np.errstate(invalid="ignore", over="ignore"):
        o = V.cross_entropy(x, w, targets, scale, teacher)
    nan = np.isnan(o["loss"])
    assert np.array_equal(np.isnan(got["loss"].f64()), nan)
    if "dx" in got:
        assert np.array_equal(np.isnan(got["dx"].f64()).all(axis=1), nan)
    rows = ~nan
    part = {k: v[rows] for k, v in o.items()}
    near = np.where(part["q"] > 0, teacher[rows] * scale, np.nan)
    with np.errstate(all="ignore"):
        near = near - np.nan_to_num(np.nanmax(np.where(np.isnan(near).all(axis=1, keepdims=True), 0.0, near), axis=1, keepdims=True))
    near = np.nan_to_num(near) / scale
    eloss, elast, edz = W.bounds(part, x[rows], w, targets[rows], dtype, scale, near)
    assert np.all(np.abs(got["loss"].f64()[rows] - part["loss"]) <= eloss)
    assert np.all(np.abs(got["lse"].f64()[rows] - part["lse"]) <= elast)
    idle = ~o["counts"]
    assert np.all(got["loss"].f64()[idle] == 0) and np.all(got["lse"].f64()[idle] == 0)
    if "dx" not in got:
        return
    dx = V.gradients(part, w, scale, 1.0)[0]
    mag = abs(scale) * (edz @ np.abs(w) + (len(w) + 8) * 2 * U32 * (np.abs(part["dz"]) @ np.abs(w)))
    gx = got["dx"].f64()
    U.close16(gx[rows], dx, dtype, mag * (1 + U.HALF_ULP[dtype]) + 4 * U32 * np.abs(dx))
    assert np.all(gx[idle] == 0)
    if nan.any():
        return
    dw = V.gradients(part, w, scale, 1.0)[1]
    mag = abs(scale) * (edz.T @ np.abs(part["x"]) + (len(x) + 24) * 2 * U32 * (np.abs(part["dz"]).T @ np.abs(part["x"])))
    U.close32(got["dw"].f64(), dw, mag + 8 * U32 * np.abs(dw))


@pytest.mark.parametrize("scale", [1.0, -0.75, 4.0, -4.0])
@pytest.mark.parametrize("dtype,kind", [("f16", "f32"), ("f16", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("k", [4, 70])
def test_masks(nnlib, k, dtype, kind, scale):
    """Entries of -inf are left out whatever the sign of the factor; entries of the type's lowest value are logits, also
    where their product with the factor passes fp32."""
    rng = np.random.default_rng(k)
    rows = 60
    x, w, targets, teacher = W.loss_inputs(rng, rows, 40, 300, dtype, k=k)
    low, high = LOWEST[kind], -LOWEST[kind]
    teacher[0, 1] = -np.inf
    teacher[1, 0], teacher[1, 2:] = -np.inf, -np.inf  # one is left
    teacher[2] = -np.inf                              # none is
    teacher[3, 1:] = low
    teacher[4] = low                                  # all alike
    teacher[5, :2], teacher[5, 2:] = low, -np.inf
    teacher[6] = high
    teacher[7, 0], teacher[7, 1:] = high, low
    teacher[8], targets[8, 1:] = low, -1
    got = W.loss_call(x, w, targets, teacher, dtype, scale, teacher_dtype=kind, dw_dtype="f32")
    check(got, x, w, targets, teacher, dtype, scale)
    check(W.loss_call(x, w, targets, teacher, dtype, scale, teacher_dtype=kind, train=False), x, w, targets, teacher, dtype, scale)


@pytest.mark.parametrize("scale", [0.5, -0.5])
def test_infinitely_high(nnlib, scale):
    """An entry of +inf: with a positive factor the row has no softmax, with a negative one no share of it; a row whose entries
    all are of that kind has no softmax either."""
    rng = np.random.default_rng(5)
    x, w, targets, teacher = W.loss_inputs(rng, 30, 24, 100, "bf16", k=3)
    teacher[4, 1] = np.inf
    teacher[9] = np.inf
    teacher[11, 0], teacher[11, 1] = np.inf, -np.inf
    got = W.loss_call(x, w, targets, teacher, "bf16", scale, dw_dtype="f32")
    check(got, x, w, targets, teacher, "bf16", scale)
