"""Plain forms, in 64 bits, of the tokens in microscaled 4-bit floating point and of their products; from the
definitions, with numpy only.

A block of 32 channels has the scale 2^e, e = floor(log2(max |x|)) - 2 (at least -127), and for each channel the number of
the value nearest to |x| / 2^e, ties to the even number, plus 8 for a sign. All of these are exact in binary64."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest(a):
    """The number of the value nearest to each a >= 0, by distance."""
    d = np.abs(np.asarray(a, dtype=np.float64)[..., None] - VALUES)
    best = d.min(axis=-1, keepdims=True)
    tie = d == best
    even = tie & (np.arange(8) % 2 == 0)
    # of two equally near numbers, which are neighbours, one is even
    return np.where(tie.sum(axis=-1) > 1, np.argmax(even, axis=-1), np.argmax(tie, axis=-1))


def quantize(x):
    """(codes uint8 [M][16 B], scales uint8 [B][M]) of the rows of a matrix of binary32 (or bfloat16) values."""
    x = np.asarray(x, dtype=np.float64)
    M, K = x.shape
    B = -(-K // 32)
    wide = np.zeros((M, 32 * B))
    wide[:, :K] = x
    blocks = wide.reshape(M, B, 32)
    with np.errstate(all="ignore"):
        top = np.max(np.abs(blocks), axis=2)
        e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)
        e = np.maximum(e, -127)
        bad = ~np.isfinite(top)
        number = nearest(np.where(bad[:, :, None], 0.0, np.ldexp(np.abs(blocks), -e[:, :, None])))
    number = np.where(bad[:, :, None], 0, number + 8 * np.signbit(blocks)).reshape(M, -1).astype(np.uint8)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    return number[:, ::2] | number[:, 1::2] << 4, np.ascontiguousarray(scales.T)


def values(codes, scales, K=None):
    """The values of codes and scales, binary64 [M][K]."""
    number = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)
    e = np.repeat(scales.T.astype(np.int64), 32, axis=1)
    v = np.ldexp(VALUES[number & 7], e - 127) * np.where(number & 8, -1.0, 1.0)
    return np.where(e == 255, np.nan, v)[:, :K]


def layer(x, w, bias=None, act="none"):
    """y[m][n] in binary64 of the values x [M][K] and w [N][K], and sum_k |x w|."""
    with np.errstate(all="ignore"):
        s = x @ w.T
        y = s if bias is None else s + bias.astype(np.float64)[None]
        if act == "relu":
            y = np.where(y < 0, 0.0, y)
        elif act == "tanh":
            y = np.tanh(y)
        return y, np.abs(x) @ np.abs(w).T
