"""The oracle's distillation where lists are padded and logits lie far apart."""
import numpy as np

from oracle import distill


def test_a_place_of_minus_infinity_adds_nothing_whatever_its_class():
    z, inf = [[0.5, -1.0, 2.0]] * 5, np.inf
    top = [[-inf, -inf], [1.0, -inf], [-inf, 1.0], [1.0, -2.0], [1.0, np.nan]]
    ids = [[3, 1], [2, 3], [2 ** 40, 2], [2, 3], [2, 3]]
    loss, grad = distill.distill(z, top, ids)
    assert loss[0] == 0 and not grad[0].any()
    r = np.exp(z[0]) / np.exp(z[0]).sum()
    for m in (1, 2):
        assert np.isclose(loss[m], -np.log(r[2])) and np.allclose(grad[m], r - [0, 0, 1])
    assert np.isnan(loss[3:]).all() and np.isnan(grad[3:]).all()


def test_bounds_stay_finite_where_the_losses_are():
    """Classes so far below the largest logit that their part of the softmax is 0 in 64 bits: the bound of a loss is that of
    some roundings of the differences, far below the loss."""
    rng = np.random.default_rng(2)
    for spread in (1.0, 1e3, 1e30):
        z, top = rng.standard_normal((20, 40)) * spread, rng.standard_normal((20, 6))
        ids = np.stack([rng.permutation(40)[:6] for _ in range(20)])
        loss, grad = distill.distill(z, top, ids, 2.0)
        bound, gbound = distill.error_bound(z, top, ids, 2.0)
        assert np.isfinite(loss).all() and np.isfinite(bound).all() and np.isfinite(gbound).all()
        assert (loss > 0.1 * spread).all() and (bound < 1e-4 * (1 + loss)).all()
        # two evaluations in 32 bits stay within it: the logits taken exactly, and rounded to binary32 differences
        d = (z - z.max(axis=1, keepdims=True)).astype(np.float32) / np.float32(2.0)
        t = (top - top.max(axis=1, keepdims=True)).astype(np.float32) / np.float32(2.0)
        e, p = np.exp(d), np.exp(t)
        p /= p.sum(axis=1, keepdims=True)
        log_p = t - np.log(np.exp(t).sum(axis=1, keepdims=True))
        log_r = np.take_along_axis(d, ids, 1) - np.log(e.sum(axis=1, keepdims=True))
        got = 4 * (p * (log_p - log_r)).sum(axis=1, dtype=np.float32)
        assert got.dtype == np.float32 and (np.abs(got - loss) <= bound).all()
