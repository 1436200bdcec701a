"""The recurrence with one channel, which has kernels of its own (a lane walks a sequence)."""
import numpy as np
import pytest

from oracle import sequence as S
from paper_2102_06725_amd import nnconv as nc

import sequence_util as U
from test_gpu_recurrence import Case

pytestmark = pytest.mark.gpu


def test_as_many_sequences_as_there_can_be(nnlib):
    """2^31 - 1 sequences of one token: the number of workgroups is counted past 32 bits.  The inputs repeat
    themselves, and so do the outputs, which are those of a call on one period."""
    t = U.torch()
    n, period = 2 ** 31 - 1, 1 << 20
    g = t.Generator(device="cuda").manual_seed(1)
    one = [t.randn((period, 1, 1), generator=g, device="cuda").half() for _ in range(3)]
    bias = t.full((1,), 0.5, device="cuda")

    def both(n, x, f, dy):
        op = nc.GatedRecurrence(n, 1, 1)
        y, dx, df, saved, dbias = t.empty_like(x), t.empty_like(x), t.empty_like(x), op.saved(), t.empty(1, device="cuda")
        op.fwd(x, f, bias, y, saved=saved)
        op.bwd(x, f, bias, saved, dy, dx, df, dbias=dbias)
        return (y, dx, df, saved), dbias
    want, part = both(period, *one)
    many = []
    for v in one:
        w = t.empty((n, 1, 1), dtype=v.dtype, device="cuda")
        for at in range(0, n, period):
            w[at:at + period] = v[:n - at]
        many.append(w)
    got, dbias = both(n, *many)
    for a, b in zip(got, want):
        a, b = a.view(-1), b.view(-1)
        assert a.numel() == n
        for at in range(0, n, period):
            assert bool((a[at:at + period] == b[:n - at]).all()), at
    # sums in fp32, at most 2^15 + 2^9 terms one after the other
    terms = float(want[2].double().abs().sum()) * (n / period)
    assert abs(float(dbias) - float(part.double()) * (n / period)) <= (2 ** 15 + 2 ** 9) * 2.0 ** -24 * terms + 2.0 ** -11 * terms / period ** 0.5


KINDS = [
    # around the stretches of saved states, and several of them
    dict(n=3, t=2, dtype="bf16"), dict(n=3, t=6, dtype="f16"), dict(n=2, t=7, dtype="f16"), dict(n=3, t=63, dtype="f16"),
    dict(n=3, t=64, dtype="bf16"), dict(n=3, t=65, dtype="f16"), dict(n=2, t=129, dtype="f16", pad=2, pady=3), dict(n=1, t=1000, dtype="f16"),
    dict(n=2, t=1003, dtype="bf16", pad=7, shift=1),
    # without g, without bias, without carried states
    dict(n=3, t=130, dtype="f16", with_g=False), dict(n=3, t=130, dtype="bf16", with_bias=False), dict(n=2, t=300, dtype="f16", carry=False),
    dict(n=2, t=300, dtype="f16", with_g=False, with_bias=False, carry=False, pad=1),
    # more sequences than a workgroup, and the last one alone in its own
    dict(n=65, t=70, dtype="f16"), dict(n=64, t=66, dtype="f16"), dict(n=130, t=17, dtype="bf16", pad=1), dict(n=600, t=3, dtype="f16"),
    # lengths: empty, one, on the edges of a stretch, past the end, below zero
    dict(n=9, t=200, dtype="f16", lengths=[0, 1, 63, 64, 65, 128, 200, 777, -5]),
    dict(n=4, t=1, dtype="f16", lengths=[0, 1, 2, -1]), dict(n=2, t=90, dtype="bf16", lengths=[0, 0], with_g=False),
    dict(n=66, t=100, dtype="f16", lengths=[(37 * i) % 103 for i in range(66)]),
    dict(n=2, t=0, dtype="f16"),
]
ids = lambda k: "-".join("%s%s" % (p, v if not isinstance(v, list) or len(v) < 10 else "many") for p, v in k.items()).replace(" ", "")  # noqa: E731


@pytest.mark.parametrize("kw", KINDS, ids=ids)
@pytest.mark.parametrize("in_place", [False, True])
def test_against_oracle(nnlib, kw, in_place):
    c = Case(c=1, seed=21, **kw)
    c.check(in_place=in_place and c.h0 is not None, old=np.array([0.75]) if in_place else None)


def test_gradients_against_differences(nnlib):
    """The sum of w y + u h_t moves with x, f, g, bias and h0 as the gradients say, by central differences of the
    oracle's forward pass in 64 bits."""
    c = Case(3, 90, 1, "f16", lengths=[90, 0, 65], seed=22)
    c.forward()
    dx, df, dg, dh0, dbias, _ = c.backward()

    def loss(**new):
        k = {v: new.get(v, getattr(c, v)) for v in ("x", "f", "g", "bias", "h0")}
        y, h = S.recurrence_fwd(k["x"], k["f"], k["bias"], k["g"], c.lengths, k["h0"])
        return (c.dy * y).sum() + (c.dht * h[:, -1]).sum()
    e = 1e-5
    rng = np.random.default_rng(5)
    for name, grad, scale in (("x", dx, 1), ("f", df, 1), ("g", dg, 1), ("h0", dh0, 1), ("bias", dbias, 4.0)):
        v = getattr(c, name)
        for _ in range(6):
            way = rng.standard_normal(v.shape)
            want = (loss(**{name: v + e * way}) - loss(**{name: v - e * way})) / (2 * e)
            terms = grad * scale * way
            # each gradient is one rounding to 11 bits from its value, and fp32 arithmetic's share; a central difference of a
            # function whose third derivatives are of its size is off by its size times e^2, and by 1e-16 / e
            assert abs(terms.sum() - want) <= 2.0 ** -10 * np.abs(terms).sum() + 1e-6


def test_infinities_and_nans(nnlib):
    """They go forward in their own sequence, and backward in the gradients, and nowhere else."""
    c = Case(70, 150, 1, "bf16", with_g=False, seed=23)
    c.x[3, 70] = np.inf
    c.x[66, 10] = -np.inf
    c.f[5, 149] = np.nan
    y, ht = c.forward()
    assert np.all(y[3, 70:] == np.inf) and np.isfinite(y[3, :70]).all() and ht[3] == np.inf
    assert np.all(y[66, 10:] == -np.inf) and np.isfinite(y[66, :10]).all() and ht[66] == -np.inf
    assert np.isnan(y[5, 149]).all() and np.isfinite(y[5, :149]).all() and np.isnan(ht[5]).all()
    rest = np.delete(np.arange(70), [3, 5, 66])
    assert np.isfinite(y[rest]).all() and np.isfinite(ht[rest]).all()
    c = Case(70, 150, 1, "bf16", with_g=False, seed=23)
    c.forward()
    c.dy[4, 100] = np.inf
    dx, df, _, dh0, dbias, flag = c.backward()
    assert np.all(dx[4, :101] == np.inf) and np.isfinite(dx[4, 101:]).all() and dh0[4] == np.inf
    assert np.isfinite(dx[np.delete(np.arange(70), 4)]).all()
    assert not np.isfinite(dbias).any() and flag == 1
