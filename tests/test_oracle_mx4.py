"""The oracle's 4-bit tokens, pinned by hand-derived cases."""
import numpy as np
import pytest

from oracle import mx4


def _one(*x):
    codes, scales = mx4.quantize(np.array([x], dtype=np.float32))
    number = np.stack([codes & 15, codes >> 4], axis=2).reshape(-1)
    return list(number[:len(x)]), int(scales[0, 0])


def test_hand_derived_blocks():
    # the largest, 6, lies in [4, 8): scale 1
    assert _one(6.0, -6.0, 0.5, 1.0, -1.5, 2.0, 3.0, 4.0) == ([7, 15, 1, 2, 11, 4, 5, 6], 127)
    # 1 is scaled to 4
    assert _one(1.0, 0.125, -0.25) == ([6, 1, 10], 125)
    # what lies above 6 becomes 6
    assert _one(7.75, 5.1) == ([7, 7], 127)


def test_ties_go_to_even_numbers():
    assert _one(4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)[0] == [6, 0, 2, 2, 4, 4, 6, 6]
    assert _one(4.0, 0.26, 0.74, 1.26, 1.74, 2.51, 3.49, 5.01)[0] == [6, 1, 1, 3, 3, 5, 5, 7]


def test_zeros_signs_and_small_blocks():
    assert _one(0.0, -0.0) == ([0, 8], 0)
    assert _one(4.0, -0.01) == ([6, 8], 127)
    # 2^-126: e would be -128, and is -127: 2^-126 / 2^-127 = 2
    assert _one(2.0 ** -126) == ([4], 0)
    assert _one(2.0 ** -149, 2.0 ** -127) == ([0, 2], 0)
    assert _one(2.0 ** 127) == ([6], 252)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_blocks_that_are_no_numbers(bad):
    x = np.ones((2, 70), dtype=np.float32)
    x[1, 40] = bad
    codes, scales = mx4.quantize(x)
    assert scales.tolist() == [[125, 125], [125, 255], [125, 125]]
    assert not codes[1, 16:32].any()
    v = mx4.values(codes, scales, 70)
    assert np.array_equal(v[0], np.ones(70)) and np.array_equal(np.isnan(v[1]), (np.arange(70) // 32) == 1)


def test_values_are_nearest_and_padding_is_zero():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 45)).astype(np.float32)
    codes, scales = mx4.quantize(x)
    assert codes.shape == (5, 32) and scales.shape == (2, 5)
    v = mx4.values(codes, scales)
    assert not v[:, 45:].any() and not codes[:, 23:].any()
    # no other number of the same block is nearer
    all_values = np.concatenate([mx4.VALUES, -mx4.VALUES])
    for m in range(5):
        for k in range(45):
            s = 2.0 ** (int(scales[k // 32, m]) - 127)
            assert abs(v[m, k] - x[m, k]) == np.min(np.abs(all_values * s - x[m, k]))


def test_layer():
    x, w = np.array([[1.0, -2.0]]), np.array([[3.0, 1.0], [0.5, 4.0]])
    y, size = mx4.layer(x, w, np.array([0.0, 0.5]))
    assert y.tolist() == [[1.0, -7.0]] and size.tolist() == [[5.0, 8.5]]
    assert mx4.layer(x, w, np.array([0.0, 0.5]), "relu")[0].tolist() == [[1.0, 0.0]]
