"""Pins of the oracle's clipping where the norm or the bound is no finite number."""
import numpy as np
import pytest

from oracle import tokens

INF = float("inf")


@pytest.mark.parametrize("element,bound,factor", [(1.0, INF, 1.0), (INF, INF, 1.0), (-INF, INF, 1.0), (INF, 2.0, 0.0),
                                                  (float("nan"), INF, float("nan")), (float("nan"), 2.0, float("nan"))])
def test_clip_without_finite_numbers(element, bound, factor):
    norm, (out, other) = tokens.clip([np.array([element, 3.0]), np.array([-4.0])], bound)
    with np.errstate(invalid="ignore"):
        want = np.array([element, 3.0]) * np.float64(factor)
    assert np.array_equal(other, [-4.0 * factor], equal_nan=True)
    assert np.array_equal(out, want, equal_nan=True)
