"""Distillation in the calls that the sizes and layouts of test_gpu_distill.py leave out.  Bounds as there, finite wherever
the expected values are."""
import numpy as np
import pytest

from oracle import distill as oracle
from paper_1508_06904_amd import dss
from tests.test_gpu_distill import _check, _dev, _inputs, _np

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------- sums of few classes and of many places
# Maps of up to 128 classes. Their sums have one term of 1 (of each 32) and others a little under u = 2^-24, half a last place
# below 1's next number: one after the other, each of them would be rounded away.

S = -16.643                              # exp(S) = 0.993 u


@pytest.mark.parametrize("C", [32, 64, 96, 128])
def test_the_classes_sum_keeps_small_terms(C):
    """r's sum is C / 32 (1 + 31 exp(S)).  Adding 32 terms by halves and C / 32 such sums one after the other rounds 5 + C / 32 - 1
    times, each by at most u of the sum; the logarithm is within 2 u of its value; exp(S) is off by less than 60 u of
    itself. The loss, log sum, has no other rounding (p = 1, the difference is 0): 5 + 3 + 2 log 4 + 1 < 12 u. The gradient of
    an unlisted class of logit 0 is 1 / sum, a division and a product more: 5 + 3 + 2 + 1 < 12 u of it."""
    z = np.full((70, C), S, dtype=np.float32)
    z[:, ::32] = 0
    top, ids = np.zeros((70, 1), dtype=np.float32), np.zeros((70, 1), dtype=np.int64)
    losses, grad = dss.distill(_dev(z.T.copy()).t(), _dev(top), _dev(ids))
    want, wgrad = oracle.distill(z, top, ids)
    assert np.abs(_np(losses) - want).max() <= 12 * U, np.abs(_np(losses) - want).max() / U
    if C > 32:
        off = np.abs(_np(grad)[:, 32] / wgrad[:, 32] - 1)
        assert off.max() <= 12 * U, off.max() / U


@pytest.mark.parametrize("k", [30, 100, 128, 600, 1024])
def test_a_lists_sum_keeps_small_terms(k):
    """Two classes of equal logits, the first listed with weight 1 and the other one k - 1 times with exp(S): with e = (k - 1) exp(S),
    the loss is log 2 - log(1 + e) + e S / (1 + e). Places are added 8 by halves, 8 such sums one after the other, and then these:
    d = 3 + min(7, k / 8) + k / 64 roundings, each by at most u of the sum, in sum_p and in the sum of p, whose rounding counts log 2 times;
    p rounds 3 times more, and the two logarithms by 2 u of log 2 and of e. Beside (d + 0.7 (d + 3) + 2 + 3) u there are
    only terms of e u. Without them the loss would be off by e, more than that."""
    top = np.full((70, k), S, dtype=np.float32)
    top[:, 0] = 0
    ids = np.ones((70, k), dtype=np.int64)
    ids[:, 0] = 0
    z = np.zeros((70, 2), dtype=np.float32)
    losses, _ = dss.distill(_dev(z.T.copy()).t(), _dev(top), _dev(ids))
    want, _ = oracle.distill(z, top, ids)
    d = 3 + min(7, k // 8) + k // 64
    bound = (d + 0.7 * (d + 3) + 5) * U
    assert (k - 1) * np.exp(S) > bound
    assert np.abs(_np(losses) - want).max() <= bound, (np.abs(_np(losses) - want).max() / U, bound / U)


# ---------------------------------------------------------------------------- places of logit -infinity

SIZES = [(70, 4, 2), (70, 64, 8), (70, 600, 8), (70, 600, 130), (70, 3000, 8), (3, 20000, 16), (3, 90000, 16), (3, 140001, 16)]


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,k", SIZES)
def test_a_place_of_minus_infinity_adds_nothing_whatever_its_class(M, C, k, dtype, layout):
    """Lists padded with a class that there is not and -infinity: alone they leave nothing to learn, beside others they
    do not count. With any other logit such a class still makes its position NaN."""
    import torch
    z, top, ids = _inputs(M, C, k, layout, dtype)
    inf = float("inf")
    ids[:, 0].clamp_(min=0)
    short = top.clone(), ids.clone()
    short[1][:, 1:] = -1
    top[:, 1:], ids[:, 1:] = -inf, C
    ids[:, k - 1] = 2 ** 40
    losses, grad = dss.distill(z, top, ids, temperature=1.5)
    _check(losses, grad, z, *short, T=1.5)
    some = z.clone(memory_format=torch.preserve_format)
    some[0] = float("nan")
    top[0], ids[0] = -inf, C
    top[1, 1], top[2, k - 1] = -1.0, float("nan")
    losses, grad = dss.distill(some, top, ids, temperature=1.5)
    assert float(losses[0]) == 0 and not bool(grad[0].any())
    assert bool(torch.isnan(losses[1:3]).all()) and bool(torch.isnan(grad[1:3]).all())
    _check(losses[3:], grad[3:], z[3:], short[0][3:], short[1][3:], T=1.5) if M > 3 else None
    want, wgrad = oracle.distill(_np(some), _np(top), ids.cpu().numpy(), 1.5)
    assert np.array_equal(np.isnan(want), _np(torch.isnan(losses)) != 0)
    assert np.array_equal(np.isnan(wgrad), _np(torch.isnan(grad)) != 0)


# ---------------------------------------------------------------------------- classes far below the largest logit

@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,k", [(70, 40, 6), (70, 300, 6), (70, 300, 130), (70, 3000, 6), (3, 20000, 6), (3, 70001, 6), (3, 140000, 6)])
@pytest.mark.parametrize("spread", [100.0, 1000.0, 1e30])
def test_losses_of_classes_far_below(M, C, k, dtype, layout, spread):
    z, top, ids = _inputs(M, C, k, layout, dtype, spread=spread)
    for T in (1.0, 4.0):
        losses, grad = dss.distill(z, top, ids, temperature=T)
        want, _ = oracle.distill(_np(z), _np(top), ids.cpu().numpy(), T)
        bound, gbound = oracle.error_bound(_np(z), _np(top), ids.cpu().numpy(), T)
        assert np.isfinite(want).all() and np.isfinite(bound).all() and np.isfinite(gbound).all()
        assert (bound <= 1e-3 * (1 + np.abs(want))).all()
        _check(losses, grad, z, top, ids, T=T)


# ---------------------------------------------------------------------------- the gradient over the logits

@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,k", [(65, 7, 3), (67, 64, 8), (130, 500, 9), (40, 300, 130), (130, 2500, 9), (5, 30000, 20), (3, 140001, 20)])
def test_beside_logits_that_their_gradient_is_written_over_nothing_changes(M, C, k, dtype, layout):
    import torch
    z, top, ids = _inputs(M, C, k, layout, dtype)
    want, wgrad = dss.distill(z, top, ids, temperature=1.5)
    rows, cols = (C, M) if layout == "map" else (M, C)
    wide = torch.full((rows + 2, cols + 5), -77.0, dtype=z.dtype, device="cuda")
    inner = wide[1:rows + 1, 3:3 + cols]
    over = inner.t() if layout == "map" else inner
    over.copy_(z)
    losses, grad = dss.distill(over, top, ids, temperature=1.5, grad=over)
    assert grad is over
    _check(losses, grad, z, top, ids, T=1.5)
    bound, gbound = oracle.error_bound(_np(z), _np(top), ids.cpu().numpy(), 1.5)
    assert (np.abs(_np(losses) - _np(want)) <= 2 * bound).all()
    inner.fill_(-77)
    assert bool((wide == -77).all())
