"""Pins of the oracle's 8-bit tokens, products and gradient clipping: cases small enough to
work out by hand, and properties the definitions imply."""
import numpy as np
import pytest

from oracle import tokens


def test_codes_by_hand():
    """scale = 254/127 = 2 exactly: halves of odd numbers are ties and go to the even code."""
    x = np.array([[254, 1, 3, 5, -1, -3, -254, 0], [0] * 8], dtype=np.float32)
    q, s = tokens.quantize(x)
    assert s.tolist() == [2.0, 0.0]
    assert q.tolist() == [[127, 0, 2, 2, 0, -2, -127, 0], [0] * 8]


def test_tokens_that_are_no_numbers_stay_alone():
    x = np.array([[1, np.nan], [np.inf, 1], [-np.inf, 0], [127, -127]], dtype=np.float32)
    q, s = tokens.quantize(x)
    assert np.isnan(s[:3]).all() and s[3] == 1 and not q[:3].any() and q[3].tolist() == [127, -127]
    y, _ = tokens.layer(q, s, np.array([[1, 2]], dtype=np.int8), np.ones(1, np.float32), act="relu")
    assert np.isnan(y[:3]).all() and y[3, 0] == 0


def test_smallest_and_largest_tokens():
    tiny, big = np.float32(1e-45), np.float32(3.4e38)
    q, s = tokens.quantize(np.array([[tiny, -tiny], [190 * tiny, tiny], [big, -big]], dtype=np.float32))
    assert s[0] == 0 and not q[0].any()              # the scale underflows
    assert s[1] == tiny and q[1].tolist() == [127, 1]  # 190 / 127 of the smallest number rounds to it; clamped
    assert q[2].tolist() == [127, -127]


@pytest.mark.parametrize("seed", range(4))
def test_codes_are_nearest(seed):
    x = np.random.default_rng(seed).standard_normal((50, 33)).astype(np.float32)
    q, s = tokens.quantize(x)
    assert np.abs(q).max(axis=1).tolist() == [127] * 50
    assert np.all(np.abs(q * s[:, None].astype(np.float64) - x) <= s[:, None] * (0.5 + 1e-4))


def test_layer_by_hand():
    codes = np.array([[127, -127, 1]], dtype=np.int8)
    weight = np.array([[1, 1, 10], [127, -127, 0]], dtype=np.int8)
    y, p = tokens.layer(codes, np.array([0.5], np.float32), weight, np.array([2, 0.25], np.float32),
                        np.array([-11, 1], np.float32), "relu")
    assert y.tolist() == [[0.0, 1 + 0.125 * 32258]] and p.tolist() == [[10.0, 0.125 * 32258]]


def test_clip_by_hand():
    norm, out = tokens.clip([np.array([3.0]), np.array([]), np.array([[0.0, -4.0]])], 1.0)
    assert norm == 5.0
    assert abs(out[0][0] - 3 / (5 + 1e-6)) < 1e-15 and out[1].size == 0
    norm, out = tokens.clip([np.array([3.0, 4.0])], 10.0)
    assert out[0].tolist() == [3.0, 4.0]
    norm, out = tokens.clip([np.array([np.inf, 1.0])], 1.0)
    assert norm == np.inf and np.isnan(out[0][0]) and out[0][1] == 0
