"""AdamW where sqrt(v) lies at the ends of fp32's range: the smallest and the largest gradients without an eps.

From moments of zero the first step is lr * sign(g), whatever the size of g.  With u = 2^-24 the change is off by
24 u (as in the operator's own tests) and by what v loses: half a unit of the smallest subnormals, 2^-150, in v itself and
as much in its correction by 1 / (1 - beta2), half of which reaches the root."""
import numpy as np
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

pytestmark = pytest.mark.gpu
f32 = lambda v: float(np.float32(v))  # noqa: E731
LR, B1, B2 = f32(2e-3), f32(0.9), f32(0.999)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-30])
def test_first_step_of_any_gradient(nnlib, bits, eps):
    t = U.torch()
    # v = 0.001 g^2 from 2^-139 (subnormal) to 2^127
    size = np.exp2(np.concatenate([np.linspace(-64.5, -40.0, 2000), np.linspace(-40.0, 68.4, 2000)]))
    g = (size * np.where(np.arange(size.size) % 3 == 0, -1.0, 1.0)).astype(np.float32)
    n = g.size
    z = lambda k, d=t.float32: t.zeros(k, dtype=d, device="cuda")  # noqa: E731
    entry = dict(master=z(n), grad=t.from_numpy(g).cuda(), m=z(n), v=z(n))
    if bits == 8:
        entry.update(m=z(n, t.float8_e4m3fn), v=z(n, t.float8_e5m2), m_scale=z(-(-n // 64), t.uint8), v_scale=z(-(-n // 64), t.uint8))
    step = z(1, t.int32)
    nc.AdamW([entry]).step(step, LR, B1, B2, f32(eps))
    got = entry["master"].double().cpu().numpy()
    g = g.astype(np.float64)
    v = (1.0 - B2) * g * g
    lost = 0.5 * (2.0 ** -150 / v + 2.0 ** -150 / (v / (1.0 - B2)))
    den = np.abs(g) + f32(eps)
    want = -LR * g / den
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > LR * (24 * 2.0 ** -24 + 2 * lost)
    assert not bad.any(), "gradients from %.3g to %.3g" % (np.abs(g[bad]).min(), np.abs(g[bad]).max())
