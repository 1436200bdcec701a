"""How many bits a logit's gradient keeps, next to tokens that are much more likely."""
import numpy as np
import pytest

import sequence_util as U
import vocabulary_util as W

pytestmark = pytest.mark.gpu
U32 = W.U32


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,v", [(1, 700), (8, 2000), (64, 20000), (512, 9000)])
def test_a_rare_tokens_gradient(nnlib, rows, v, dtype):
    """Probabilities from 1 to 2^-60 in every tile.  Each row has a channel of its own with x = 1, so that the gradient of w
    is that of the logits itself.

    A probability is rounded as an exponential, to 12 bits (fp16) or 11 (bf16), and as an operand to the type's, in units
    of 2^-15.  The exponentials' arguments lie within 60 of 0 in units of log 2, with three roundings each; the rest is
    fp32.  Below 2^-30 (fp16) of the tile's largest, steps are of 2^-41 of it; below 2^-14 in fp16, an operand's are 2^-24."""
    rng = np.random.default_rng(rows + v)
    c = max(8, rows)
    w, x = np.zeros((v, c)), np.zeros((rows, c))
    x[np.arange(rows), np.arange(rows)] = 1.0
    w[:, :rows] = U.round16(dtype)(-40.0 * rng.random((v, rows)))
    w[rng.permutation(v)[::97], :rows] = 0.0  # likely ones
    label = rng.integers(0, v, rows)
    got = W.loss_call(x, w, label[:, None], None, dtype, dw_dtype="f32")["dw"].f64()
    e = np.exp(w[:, :rows])
    p = e / e.sum(axis=0)
    others = np.arange(v)[:, None] != label
    bits, store, step = (2.0 ** -11, 2.0 ** -12, 2.0 ** -40 + 2.0 ** -42) if dtype == "f16" else (2.0 ** -8, 2.0 ** -11, 2.0 ** -73)
    rel = 2 * 3 * 60 * np.log(2) * U32 + (100 + v / 8192) * U32
    bound = p * ((1 + bits) * (1 + store) * (1 + rel) - 1) + step
    bad = (np.abs(got[:, :rows] - p) > bound) & others
    assert not bad.any(), "%d, from a probability of %.3g on" % (bad.sum(), p[bad].max())
    if dtype == "bf16":  # none is lost
        assert (got[:, :rows][others] > 0).all()
    else:
        assert (got[:, :rows][others & (p > 2.0 ** -39)] > 0).all()
    assert not got[:, rows:].any()
