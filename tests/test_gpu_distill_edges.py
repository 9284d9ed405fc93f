"""Distillation in the calls that the sizes and layouts of test_gpu_distill.py leave out.  Bounds as there, finite wherever
the expected values are."""
import numpy as np
import pytest

from oracle import distill as oracle
from paper_1508_06904_amd import dss
from tests.test_gpu_distill import _check, _inputs, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


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
