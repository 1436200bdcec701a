"""The recurrence with one channel, which has kernels of its own (a lane walks a sequence)."""
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

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
