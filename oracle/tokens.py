"""Plain forms, in 64 bits, of the 8-bit tokens, of their products with 8-bit weights and of
the gradient norm and clipping; from their definitions, with numpy only.

Scales and quotients are binary32 numbers by definition, so those two divisions are numpy's
binary32 ones (correctly rounded); everything else is in binary64 or exact integers."""
from __future__ import annotations

import numpy as np


def quantize(x):
    """Codes (int8) and scales (binary32) of the rows of a binary32 matrix."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        top = np.max(np.abs(x), axis=1)
        scales = np.where(np.isfinite(top), top / np.float32(127), np.float32(np.nan)).astype(np.float32)
        live = scales > 0
        q = x / np.where(live, scales, np.float32(1))[:, None]
        q = np.where(live[:, None], np.clip(np.rint(q), -127, 127), 0)
    return q.astype(np.int8), scales


def layer(codes, scales, weight, weight_scales, bias=None, act="none"):
    """y[m][n] in binary64, and the absolute value of its product term (before bias and activation)."""
    # |sum| < 2^53: binary64 products of integers are exact
    s = codes.astype(np.float64) @ weight.astype(np.float64).T
    with np.errstate(all="ignore"):
        prod = s * weight_scales.astype(np.float64)[None] * scales.astype(np.float64)[:, None]
        y = prod if bias is None else prod + bias.astype(np.float64)[None]
        if act == "relu":
            y = np.where(y < 0, 0.0, y)
        elif act == "tanh":
            y = np.tanh(y)
    return y, np.abs(prod)


def grad_norm(grads):
    """The norm over all arrays of a list."""
    with np.errstate(all="ignore"):
        return float(np.sqrt(sum(float(np.sum(np.asarray(g, dtype=np.float64) ** 2)) for g in grads)))


def clip(grads, max_norm):
    """(norm, the scaled arrays in binary64)."""
    norm = grad_norm(grads)
    with np.errstate(all="ignore"):
        c = np.float64(max_norm) / np.float64(norm + 1e-6)
        # an infinite bound clips nothing, infinite elements included; a NaN norm stays one
        c = 1.0 if c >= 1.0 or (np.isinf(max_norm) and not np.isnan(norm)) else c
        return norm, [np.asarray(g, dtype=np.float64) * c for g in grads]
