"""The example that distils a network from a teacher's top logits and answers with its head in 4 bits, as a run of the
operators together: maps, loss and gradient, backpropagation, clipping, coding and layers."""
import importlib.util
import os

import numpy as np
import pytest

import oracle
from oracle import backward as ob
from oracle import dilate, distill as od, mx4
from paper_1508_06904_amd import dss, workloads as wl
from tests.test_gpu_backward import TOL, close

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distill_and_answer", os.path.join(ROOT, "examples", "distill_and_answer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _networks(example, size, seed):
    import torch
    rng = np.random.default_rng(seed)
    teacher, student = wl.init_layers(example.TEACHER, rng), wl.init_layers(example.BODY + example.HEAD, rng)
    return teacher, student, torch.from_numpy(wl.blob_image(rng, 3, size, size, 8)).cuda()


def _loss(layers, x, top, ids, T):
    """The example's loss in 64 bits, and the gradient of the last layer's maps."""
    out = dilate.eval_dilate(layers, x)
    z = out.reshape(out.shape[0], -1).T
    losses, grad = od.distill(z, top.T, ids.T, T, 1.0 / z.shape[0])
    return losses.sum(), grad.T.reshape(out.shape)


def test_it_runs(example):
    student, x, (top, ids), full, coded = example.main(steps=3, size=60)
    assert coded.shape == full.shape and bool(coded.isfinite().all())
    assert example.main(steps=0, size=60)[0] is not None


def test_gradients_of_the_chain(example):
    """Against backpropagation in 64 bits within the backward pass's bound, and against differences of the 64-bit loss: along a
    direction d, (L(w + h d) - L(w - h d)) / 2h is <g, d> within h^2 / 6 of a third derivative, and within what units
    and pools that change sides in between add, both far below 1 % of it at h = 1e-5 (the oracle's own gradient is held to
    1e-4 there)."""
    T = 2.0
    teacher, student, x = _networks(example, 34, 3)
    top, ids = example.ask(teacher, x, 5)
    loss, weights, biases = example.gradients(student, x, top, ids, T)
    args = x.cpu().numpy().astype(np.float64), top.cpu().numpy().astype(np.float64), ids.cpu().numpy(), T
    want, G = _loss(student, *args)
    assert abs(float(loss) - want) <= TOL * abs(want)
    gw, gb, _ = ob.dense_backward(student, args[0], G)
    for t, (a, b) in enumerate(zip(weights + biases, list(gw) + list(gb))):
        close(a.cpu().numpy().astype(np.float64), b, "tensor %d" % t)
    rng = np.random.default_rng(4)
    convs = [l for l in student if l["kind"] == "conv"]
    ds = [[np.sign(g) * rng.random(g.shape) for g in gs] for gs in (gw, gb)]

    def moved(h):
        at = iter(zip(*ds))
        layers = []
        for l in student:
            if l["kind"] == "conv":
                dw, db = next(at)
                l = dict(l, weight=l["weight"].astype(np.float64) + h * dw, bias=l["bias"].astype(np.float64) + h * db)
            layers.append(l)
        return _loss(layers, *args)[0]

    assert len(convs) == len(gw)
    h = 1e-5
    slope = (moved(h) - moved(-h)) / (2 * h)
    inner = [sum(float((np.asarray(a, np.float64) * d).sum()) for gs, dd in zip(g, ds) for a, d in zip(gs, dd))
             for g in ((gw, gb), ([w.cpu().numpy() for w in weights], [b.cpu().numpy() for b in biases]))]
    assert abs(slope - inner[0]) <= 1e-2 * abs(inner[0]) and abs(inner[1] - inner[0]) <= 2 * TOL * abs(inner[0]) * len(gw)


def test_the_head_in_4_bits(example):
    """Layer by layer against the codes' values in 64 bits: every layer is given the library's own maps, so a rounding that
    falls on the other side of a code's border in one layer is no difference in the next."""
    import torch
    from tests.test_gpu_mx4 import _check_layer
    _, student, x = _networks(example, 60, 5)
    n = len(example.HEAD)
    y = dss.Plan(student[:-n], 2, 3).eval_dense(x).flatten(1)
    for l, (codes, scales) in zip(student[-n:], example.code_head(student)):
        w, ws = mx4.quantize(l["weight"].reshape(l["cout"], l["cin"]))
        assert np.array_equal(codes.cpu().numpy(), w) and np.array_equal(scales.cpu().numpy(), ws)
        v = mx4.values(*mx4.quantize(y.t().cpu().numpy()))
        y = dss.linear_mx4(y.t(), codes, scales, bias=torch.from_numpy(l["bias"]).cuda(), act=l["act"], planar=True)
        _check_layer(y.t(), v, mx4.values(w, ws), l["bias"], l["act"])
    assert torch.equal(y.view(200, -1), example.answer(student, example.code_head(student), x).flatten(1))


def test_a_captured_step_of_loss_and_answer(example):
    """Loss, gradient, clipping's norm and the coded head in one graph, replayed on other maps with eager calls between."""
    import torch
    teacher, student, x = _networks(example, 60, 6)
    top, ids = example.ask(teacher, x, 6)
    head = example.code_head(student)
    plan, n = dss.Plan(student, 2, 3), len(example.HEAD)
    z = plan.eval_dense(x).flatten(1)
    maps = dss.Plan(student[:-n], 2, 3).eval_dense(x).flatten(1)
    first, second = student[-2:]
    b1, b2 = (torch.from_numpy(l["bias"]).cuda() for l in (first, second))
    zs, ms = torch.empty_like(z), torch.empty_like(maps)

    def step(z, maps):
        losses, grad = dss.distill(z.t(), top.t(), ids.t(), temperature=2.0)
        norm = dss.grad_norm([grad.t()])
        y = dss.linear_mx4(maps.t(), *head[0], bias=b1, act=first["act"], planar=True)
        return losses, grad, norm, dss.linear_mx4(y.t(), *head[1], bias=b2, act=second["act"], planar=True)

    zs.copy_(z)
    ms.copy_(maps)
    step(zs, ms)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(zs, ms)
    for turn in range(4):
        zs.copy_(z * (1 + turn) - turn)
        ms.copy_(maps * (2 - turn))
        want = step(zs.clone(), ms.clone())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn


def test_receptive_fields_agree(example):
    rng = np.random.default_rng(0)
    assert oracle.receptive_field(wl.init_layers(example.TEACHER, rng)) == oracle.receptive_field(
        wl.init_layers(example.BODY + example.HEAD, rng))
