"""Rows that do not count have gradients of 0 whatever w holds, and whatever the gradients are scaled by."""
import numpy as np
import pytest

import sequence_util as U
import vocabulary_util as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [None, 3])
@pytest.mark.parametrize("rows,c,v,dtype", [
    (600, 520, 20000, "bf16"),  # whole tiles, lines of 16 bytes
    (90, 41, 500, "f16"),       # odd channels
    (20, 24, 9001, "bf16"),     # a split reduction
    (33, 8, 70, "f16")])
def test_infinities_in_w(nnlib, rows, c, v, dtype, k):
    rng = np.random.default_rng(rows)
    x, w, targets, teacher = W.loss_inputs(rng, rows, c, v, dtype, k=k, pad=0.4)
    idle = ~((targets >= 0) & (targets < v)).any(axis=1)
    assert idle.any() and not idle.all()
    w[v // 2, c // 2], w[v - 1, c - 1], w[0, 0] = np.inf, np.nan, -np.inf
    got = W.loss_call(x, w, targets, teacher, dtype)
    dx = got["dx"].f64()
    assert not dx[idle].any() and np.isnan(dx[~idle]).any(axis=1).all()
    assert not got["loss"].f64()[idle].any() and not got["lse"].f64()[idle].any()


@pytest.mark.parametrize("rows,c,v", [(300, 64, 2000), (31, 13, 700)])
@pytest.mark.parametrize("k", [None, 2])
def test_a_batch_of_padding(nnlib, rows, c, v, k):
    """No row counts: nothing of w or x is met, no gradient and no flag."""
    t = U.torch()
    rng = np.random.default_rng(c)
    x, w, targets, teacher = W.loss_inputs(rng, rows, c, v, "bf16", k=k)
    targets[:], x[:] = -1, np.nan
    w[::3] = np.inf
    flag = t.zeros(1, dtype=t.int32, device="cuda")
    got = W.loss_call(x, w, targets, teacher, "bf16", flag=flag, dw_dtype="f32")
    for key in ("loss", "lse", "dx", "dw"):
        assert not got[key].f64().any(), key
    assert int(flag) == 0
    # a mean over no rows: the factor is infinite
    got = W.loss_call(x, w, targets, teacher, "bf16", grad_scale=np.inf, want_dw=False, flag=flag)
    assert not got["dx"].f64().any() and int(flag) == 0
