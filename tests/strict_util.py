"""Comparisons that hold infinities to their place and sign, and NaNs to theirs."""
from __future__ import annotations

import numpy as np

import sequence_util as U


def nonfinite(got, ref, top=None):
    """Where both are finite.  A NaN has to meet a NaN and an infinity the same infinity; with `top`, the type's largest
    value, a result may also be infinite where the reference rounds past it, with the reference's sign."""
    assert got.shape == ref.shape
    assert np.array_equal(np.isnan(got), np.isnan(ref)), "NaNs elsewhere"
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), "an infinity is lost or has the other sign"
    over = np.isinf(got) & ~inf
    assert top is not None or not over.any(), "infinite where the reference is not"
    if over.any():
        assert np.all(np.abs(ref[over]) >= top) and np.all(np.sign(got[over]) == np.sign(ref[over])), "overflow"
    return np.isfinite(got) & np.isfinite(ref)


def within(got, ref, bound, both):
    bound = np.broadcast_to(bound, ref.shape)[both]
    err = np.abs(got[both] - ref[both])
    assert not (err > bound).any() and not np.isnan(bound).any(), "worst %.3g of its bound" % np.nanmax(err / bound)


def close16(got, ref, dtype, slack):
    """As sequence_util.close16: one rounding to the type, plus `slack`."""
    both = nonfinite(got, ref, float(U.torch().finfo(U.tdtype(dtype)).max))
    within(got, ref, U.HALF_ULP[dtype] * np.abs(ref) + U.TINY[dtype] + slack, both)


def close32(got, ref, bound):
    within(got, ref, bound, nonfinite(got, ref))


def finite(v):
    """Magnitudes for bounds: what is not finite counts as 0."""
    return np.where(np.isfinite(v), np.abs(v), 0.0)
