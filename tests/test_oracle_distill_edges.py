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
