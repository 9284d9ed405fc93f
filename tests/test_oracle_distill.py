"""The oracle's distillation loss, pinned by hand-derived cases, closed forms and differences."""
import numpy as np

from oracle import distill


def test_one_place_is_the_cross_entropy():
    z = np.array([[1.0, 2.0, 0.5]])
    loss, grad = distill.distill(z, [[7.0]], [[1]])
    r = np.exp(z[0]) / np.exp(z[0]).sum()
    assert np.allclose(loss, -np.log(r[1])) and np.allclose(grad[0], r - [0, 1, 0])


def test_a_whole_list_of_the_same_logits_is_no_loss():
    z = np.array([[0.3, -1.0, 2.0, 0.0]])
    loss, grad = distill.distill(z, z[:, [2, 0, 3, 1]] + 5, [[2, 0, 3, 1]], T=2.0)
    assert abs(loss[0]) < 1e-15 and np.abs(grad).max() < 1e-15


def test_two_classes_by_hand():
    # p = (3/4, 1/4), r = (1/2, 1/2): KL = 3/4 log(3/2) + 1/4 log(1/2)
    loss, grad = distill.distill([[0.0, 0.0]], [[np.log(3.0), 0.0]], [[0, 1]], scale=2.0)
    assert np.allclose(loss, 2 * (0.75 * np.log(1.5) + 0.25 * np.log(0.5)))
    assert np.allclose(grad, [[2 * -0.25, 2 * 0.25]])


def test_left_out_and_empty_positions():
    z = np.array([[np.nan, 1.0]] * 4 + [[0.0, 1.0]])
    top = [[1.0, 2.0], [1.0, 2.0], [-np.inf, 2.0], [1.0, 2.0], [0.0, -np.inf]]
    ids = [[0, 1], [-1, -7], [1, -1], [0, 1], [1, 0]]
    loss, grad = distill.distill(z, top, ids, weights=[0, 1, 1, 1, 1])
    assert loss[:3].tolist() == [0, 0, 0] and not grad[:3].any() and np.isnan(loss[3]) and np.isnan(grad[3]).all()
    r = np.exp([0, 1]) / np.exp([0, 1]).sum()
    assert np.allclose(loss[4], -np.log(r[1])) and np.allclose(grad[4], [r[0], r[1] - 1])
    loss, grad = distill.distill([[0.0, 0.0]], [[1.0]], [[2]])
    assert np.isnan(loss).all() and np.isnan(grad).all()


def test_gradient_is_the_losses_difference():
    rng = np.random.default_rng(1)
    z, top = rng.standard_normal((3, 6)), rng.standard_normal((3, 4))
    ids = np.array([[0, 3, 3, 5], [1, -1, 2, 4], [5, 4, 0, 1]])    # (a class twice, an empty place)
    for T in (1.0, 2.5):
        _, grad = distill.distill(z, top, ids, T, 0.5, [1.0, 2.0, 0.25])
        for m in range(3):
            for c in range(6):
                h = np.zeros((3, 6))
                h[m, c] = 1e-5
                d = [distill.distill(z + s * h, top, ids, T, 0.5, [1.0, 2.0, 0.25])[0][m] for s in (1, -1)]
                assert abs((d[0] - d[1]) / 2e-5 - grad[m, c]) < 1e-9
