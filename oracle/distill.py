"""The plain form, in 64 bits, of the distillation from a teacher's top logits; from its definition, with numpy only, one
position at a time.

With p = softmax(t / T) over a position's places and r = softmax(z / T) over all classes,
    loss = s w T^2 sum_j p_j (log p_j - log r_{i_j}),   grad_c = s w T (r_c - sum_{j: i_j = c} p_j);
both are 0 where w is 0 or no place has a logit above -infinity."""
from __future__ import annotations

import numpy as np


def _log_softmax(v):
    top = np.max(v)
    return v - top - np.log(np.sum(np.exp(v - top)))


def distill(z, top, ids, T=1.0, scale=1.0, weights=None):
    """(losses [M], gradients [M][C]) in binary64."""
    z = np.asarray(z, dtype=np.float64)
    M, C = z.shape
    losses, grad = np.zeros(M), np.zeros((M, C))
    with np.errstate(all="ignore"):
        for m in range(M):
            w = 1.0 if weights is None else float(weights[m])
            # a place of logit -infinity adds 0, whatever its class
            used = (np.asarray(ids[m]) >= 0) & (np.asarray(top[m], dtype=np.float64) != -np.inf)
            t, i = np.asarray(top[m], dtype=np.float64)[used] / T, np.asarray(ids[m])[used]
            if w == 0 or not used.any():
                continue
            if np.any(i >= C):
                losses[m], grad[m] = np.nan, np.nan
                continue
            log_p, log_r = _log_softmax(t), _log_softmax(z[m] / T)
            p = np.exp(log_p)
            terms = [0.0 if a == 0 else a * (b - c) for a, b, c in zip(p, log_p, log_r[i])]
            g = np.exp(log_r)
            for a, c in zip(p, i):
                g[c] -= a
            losses[m], grad[m] = scale * w * T * T * np.sum(terms), scale * w * T * g
    return losses, grad


def error_bound(z, top, ids, T=1.0, scale=1.0, weights=None):
    """How far a binary32 evaluation may be from distill(): (losses [M], gradients [M][C]), for finite logits.

    u = 2^-24. An exponential of d = (v - max) / T: the difference, 1/T and their product round, so its exponent is off by
    3 u |d|, and the function by 2 u. A sum of n such, no thread adding more than n_c = 1024 + n / 256 of them:
    (n_c + 16) u, and the mean of its terms' errors. A quotient by the sum: 2 u. log r and log p: 4 u of the two
    differences, and of the logarithms' own values 2 u each beside the sums' errors.

    Beside that an exponential below the smallest normal number may count as 0 (the hardware's own power of two
    gives no smaller results): it is off by less than 2^-126, and so is its quotient by the sum, which is at least 1."""
    u, small = 2.0 ** -24, 2.0 ** -126
    z = np.asarray(z, dtype=np.float64)
    M, C = z.shape
    losses, grad = np.zeros(M), np.zeros((M, C))

    def share(v):
        d = np.abs(v - np.max(v)) / T
        log_p = _log_softmax(v / T)
        p = np.exp(log_p)
        of_sum = min(v.size, 1024) + v.size / 256 + 16 + np.sum(p * (3 * d + 2))
        return p, log_p, d, u * of_sum, u * (3 * d + 2 + 2)

    for m in range(M):
        w = abs(scale) * (1.0 if weights is None else abs(float(weights[m])))
        used = np.asarray(ids[m]) >= 0
        t, i = np.asarray(top[m], dtype=np.float64)[used], np.asarray(ids[m])[used]
        if w == 0 or not np.any(t > -np.inf):
            continue
        t, i = t[t > -np.inf], i[t > -np.inf]
        p, log_p, dt, sum_p, one_p = share(t)
        r, log_r, dz, sum_r, one_r = share(z[m])
        size = np.abs(log_p - log_r[i])      # (r itself may be 0 in 64 bits)
        logs = abs(np.log(np.sum(np.exp(-dt)))) + abs(np.log(np.sum(np.exp(-dz))))
        off = 4 * u * (dt + dz[i]) + sum_p + sum_r + 2 * u * logs + 2 * u * size
        losses[m] = w * T * T * np.sum(p * (size * (sum_p + one_p + (t.size + 8) * u) + off) + small * size)
        g = r * (sum_r + one_r)
        for a, b, c in zip(p, one_p + sum_p, i):
            g[c] += a * (b + t.size * u)
        exact = np.array(r)
        for a, c in zip(p, i):
            exact[c] -= a
        grad[m] = w * T * (g + 4 * u * np.abs(exact) + small * (1 + t.size))
    return 1.01 * losses + 1e-44, 1.01 * grad + 1e-44
