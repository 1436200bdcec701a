"""The strict comparisons refuse what they are there to refuse (mistakes planted in the values)."""
import numpy as np
import pytest

import strict_util as X

INF, NAN = np.inf, np.nan
REF = np.array([1.0, INF, -INF, NAN, 70000.0, -70000.0, 0.0])


def test_the_same_values_pass():
    X.close16(np.array([1.0, INF, -INF, NAN, INF, -INF, 0.0]), REF, "f16", 0.0)
    X.close32(REF.copy(), REF, 0.0)


@pytest.mark.parametrize("at,value", [(0, 1.01), (0, INF), (0, NAN), (1, 1.0), (1, -INF), (1, NAN), (2, INF), (2, -65504.0), (2, NAN),
                                      (3, 1.0), (3, INF), (4, -INF), (4, NAN), (4, 65504.0), (5, INF), (6, -INF), (6, NAN), (6, 1e-3)])
def test_16_bits(at, value):
    got = np.array([1.0, INF, -INF, NAN, INF, -INF, 0.0])
    got[at] = value
    with pytest.raises(AssertionError):
        X.close16(got, REF, "f16", 0.0)


@pytest.mark.parametrize("at,value", [(0, 1.01), (0, INF), (0, NAN), (1, 1.0), (1, -INF), (1, NAN), (2, INF), (2, 0.0), (3, 1.0), (3, INF),
                                      (4, INF), (5, INF), (6, NAN)])
def test_32_bits(at, value):
    got = REF.copy()
    got[at] = value
    with pytest.raises(AssertionError):
        X.close32(got, REF, 1e-3)


def test_a_bound_that_is_no_number():
    with pytest.raises(AssertionError):
        X.close32(np.array([1.0]), np.array([1.0]), np.array([NAN]))
