"""The largest factor of the logits: what a logit counts in units of log 2 has to be a number of fp32."""
import numpy as np
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U
import vocabulary_util as W

TOP = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("scale,status", [(2.0 ** 127, nc.NNCONV_OK), (-2.0 ** 127, nc.NNCONV_OK), (1.25 * 2.0 ** 127, nc.NNCONV_ERR_UNSUPPORTED),
                                          (TOP, nc.NNCONV_ERR_UNSUPPORTED), (-TOP, nc.NNCONV_ERR_UNSUPPORTED)])
def test_refused(nnlib, scale, status):
    d = nc.nnconv_xent_desc(4, 16, 9, nc.NNCONV_F16, 1, nc.NNCONV_F32, scale)
    for pass_ in (nc.NNCONV_FWD, nc.NNCONV_DGRAD):
        assert nc.nnconv_xent_workspace_size(d, pass_)[0] == status
    none = nc.nnconv_xent_desc(0, 16, 9, nc.NNCONV_F16, 1, nc.NNCONV_F32, scale)
    assert nc.nnconv_xent_fwd(none, None, None, None, None, None, None, None, 0, None) == status
    assert nc.nnconv_xent_train(none, None, None, None, None, 1.0, None, None, None, None, None, nc.NNCONV_F32, 1.0, 0, None, None, 0,
                                None) == status


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** 127, -2.0 ** 127])
def test_the_largest(nnlib, scale):
    """Equal tokens share the probability, and all others have none."""
    rng = np.random.default_rng(1)
    rows, c, v = 20, 8, 300
    w, x = np.zeros((v, c)), np.zeros((rows, c))
    w[:, 0] = np.sign(scale) * 2.0 ** -60 * rng.integers(0, 4, v)
    x[:, 0] = 2.0 ** -60
    best = np.flatnonzero(np.sign(scale) * w[:, 0] == 3 * 2.0 ** -60)
    label = rng.choice(best, rows)
    got = W.loss_call(x, w, label[:, None], None, "bf16", scale, dw_dtype="f32")
    # 40 terms at most, with an exponential of 1 each
    assert np.all(np.abs(got["loss"].f64() - np.log(len(best))) <= 100 * W.U32)
    z = 3 * 2.0 ** 7
    assert np.all(np.abs(got["lse"].f64() - z - np.log(len(best))) <= 100 * W.U32 + 4 * W.U32 * z)
    dz = np.zeros((rows, v))
    dz[:, best] = 1.0 / len(best)
    dz[np.arange(rows), label] -= 1.0
    # exponentials and operands are rounded to 11 and 8 bits
    dw = scale * dz.T @ x
    mag = abs(scale) * (np.abs(dz).T @ np.abs(x))
    U.close32(got["dw"].f64(), dw, (2.0 ** -8 + 2.0 ** -10 + 400 * W.U32) * mag)
