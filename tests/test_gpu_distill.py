"""Distillation from a teacher's top logits against the oracle's 64-bit form, within the oracle's bound for a binary32
evaluation; a bfloat16 gradient rounds once more (2^-8 of its value)."""
import numpy as np
import pytest

from oracle import distill as oracle
from paper_1508_06904_amd import dss

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _np(t):
    return t.float().cpu().numpy()


def _inputs(M, C, k, layout="rows", dtype="f32", seed=0, pad=0, spread=3.0, repeat=False):
    """(logits as a view, top logits, ids) on the GPU; a few empty places, with `repeat` classes more than once."""
    import torch
    rng = np.random.default_rng([seed, M, C, k])
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    z = _dev((rng.standard_normal((M, C)) * spread).astype(np.float32)).to(dt)
    wide = torch.full((C, M + pad) if layout == "map" else (M, C + pad), float("nan"), dtype=dt, device="cuda")
    if layout == "map":
        wide[:, :M] = z.t()
        z = wide[:, :M].t()
    else:
        wide[:, :C] = z
        z = wide[:, :C]
    top = (rng.standard_normal((M, k)) * 2).astype(np.float32)
    ids = np.stack([rng.choice(C, k, replace=repeat or k > C) for _ in range(M)]).astype(np.int64)
    ids[rng.random((M, k)) < 0.1] = -1
    return z, _dev(top), _dev(ids)


def _check(losses, grad, z, top, ids, T=1.0, scale=1.0, weights=None):
    w = None if weights is None else weights.cpu().numpy()
    args = (_np(z), _np(top), ids.cpu().numpy(), T, scale, w)
    want, wgrad = oracle.distill(*args)
    bound, gbound = oracle.error_bound(*args)
    got = losses.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], bound[bad][:5])
    if grad is None:
        return
    import torch
    assert grad.shape == z.shape and grad.dtype == z.dtype
    if z.dtype == torch.bfloat16:
        gbound = gbound + 2.0 ** -8 * (np.abs(wgrad) + gbound) + 2.0 ** -134
    got = _np(grad).astype(np.float64)
    bad = ~(np.abs(got - wgrad) <= gbound)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], wgrad[bad][:5], gbound[bad][:5])


SIZES = [(1, 1, 1), (1, 2, 1), (1, 4, 2), (3, 2, 2), (5, 3, 3), (64, 16, 4), (65, 17, 5), (257, 33, 8), (300, 64, 8), (70, 65, 9),
         (129, 100, 33), (40, 128, 128), (33, 257, 16), (67, 500, 40), (66, 1000, 16), (20, 1025, 64), (10, 2049, 100),
         (5, 4096, 257), (3, 9001, 1000), (2, 20000, 1024), (7, 33000, 64), (2, 70001, 31), (1, 131071, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout,pad", [("rows", 0), ("rows", 3), ("map", 0), ("map", 5)])
@pytest.mark.parametrize("M,C,k", SIZES)
def test_losses_and_gradients(M, C, k, layout, pad, dtype):
    import torch
    z, top, ids = _inputs(M, C, min(k, 1024), layout, dtype, pad=pad)
    losses, grad = dss.distill(z, top, ids)
    _check(losses, grad, z, top, ids)
    # the loss alone, the other types of lists, a temperature and weights
    weights = torch.rand(M, device="cuda") - 0.3
    weights[::3] = 0
    half = top.to(torch.bfloat16)
    kw = dict(temperature=2.5, scale=0.37, weights=weights)
    losses, none = dss.distill(z, half, ids.int(), with_grad=False, **kw)
    assert none is None
    _check(losses, None, z, half, ids, 2.5, 0.37, weights)
    again, grad = dss.distill(z, half, ids.int(), **kw)
    _check(again, grad, z, half, ids, 2.5, 0.37, weights)
    assert not bool(grad[::3].any()) and not bool(again[::3].any())


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(9, 2, 3), (70, 5, 16), (300, 40, 64), (21, 300, 64), (8, 5000, 700), (3, 40000, 1024)])
def test_classes_more_than_once(M, C, k, layout):
    z, top, ids = _inputs(M, C, k, layout, repeat=True)
    ids[0] = ids[0, 0].clamp(min=0)
    losses, grad = dss.distill(z, top, ids)
    _check(losses, grad, z, top, ids)


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,k", [(70, 4, 2), (70, 64, 8), (66, 600, 8), (5, 20000, 16), (3, 90000, 16)])
def test_positions_that_are_left_out(M, C, k, dtype, layout):
    """Weight 0, empty lists and lists of -infinity: exact zeros, whatever the logits."""
    import torch
    z, top, ids = _inputs(M, C, k, layout, dtype)
    weights = torch.ones(M, device="cuda")
    keep = z.clone()
    weights[0] = 0
    z[0] = float("nan")
    ids[1] = -1
    z[1, 0] = float("inf")
    top[2] = -float("inf")
    z[2] = -float("inf")
    top[M - 1, 0] = float("nan")
    ids[M - 1, 0] = -5                                  # (an empty place's logit does not count)
    losses, grad = dss.distill(z, top, ids, weights=weights)
    assert not bool(losses[:3].any()) and not bool(grad[:3].any())
    keep[:3] = 0
    top[M - 1, 0] = 0
    _check(losses, grad, keep, top, ids, weights=weights)


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(70, 4, 2), (70, 64, 8), (66, 600, 8), (6, 20000, 16), (6, 90000, 16)])
def test_infinities_and_nan(M, C, k, layout):
    import torch
    z, top, ids = _inputs(M, C, k, layout)
    ids.clamp_(min=0)
    ids[:, 1] = (ids[:, 0] + 1) % C
    inf = float("inf")
    z[0, ids[0, 0]] = -inf                              # a class that the teacher wants: an infinite loss
    top[1, 0], z[1, ids[1, 0]] = -inf, -inf             # one that it does not: adds nothing
    z[2, C // 2] = float("nan")
    z[3] = -inf
    z[4, C - 1] = inf
    top[5, 1] = float("nan")
    if k > 2:
        ids[1, 2:] = -1
    losses, grad = dss.distill(z, top, ids)
    want, wgrad = oracle.distill(_np(z), _np(top), ids.cpu().numpy())
    assert float(losses[0]) == inf and bool(torch.isfinite(grad[0]).all())
    assert bool(torch.isnan(losses[2:6]).all()) and bool(torch.isnan(grad[2:5]).all())
    assert np.array_equal(np.isnan(_np(grad)), np.isnan(wgrad))
    for m in {1, M - 1} - {5}:
        assert abs(float(losses[m]) - want[m]) < 1e-5 * max(1, abs(want[m]))
        assert np.abs(_np(grad[m]) - wgrad[m]).max() < 1e-5


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(70, 4, 2), (70, 64, 8), (66, 600, 8), (3, 20000, 16), (3, 90000, 16)])
def test_a_class_that_there_is_not_spoils_its_position_only(M, C, k, layout):
    import torch
    z, top, ids = _inputs(M, C, k, layout)
    ids[1, k - 1] = C
    ids[2, 0] = 2 ** 40
    losses, grad = dss.distill(z, top, ids)
    assert bool(torch.isnan(losses[1:3]).all()) and bool(torch.isnan(grad[1:3]).all())
    keep = [0] + list(range(3, M))
    _check(losses[keep], grad[keep], z[keep], top[keep], ids[keep])


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,k", [(65, 7, 3), (67, 64, 8), (130, 500, 9), (5, 30000, 20), (3, 140001, 20)])
def test_the_gradient_over_the_logits(M, C, k, dtype, layout):
    import torch
    z, top, ids = _inputs(M, C, k, layout, dtype, pad=2)
    want, wgrad = dss.distill(z, top, ids, temperature=1.5)
    buf = z.clone(memory_format=torch.preserve_format)
    losses, grad = dss.distill(z, top, ids, temperature=1.5, grad=z)
    assert grad is z and torch.equal(losses, want) and torch.equal(grad, wgrad)
    assert buf.shape == z.shape


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(1, 5, 2), (67, 64, 8), (130, 500, 9), (5, 30000, 20), (5, 140000, 20)])
def test_gradients_and_lists_in_wider_buffers(M, C, k, layout):
    """Strides of every operand; beside the gradient nothing is written."""
    import torch
    z, top, ids = _inputs(M, C, k, layout, pad=7)
    rows, cols = (C, M) if layout == "map" else (M, C)
    gb = torch.full((rows + 2, cols + 5), -77.0, device="cuda")
    out = gb[1:rows + 1, 2:2 + cols]
    grad = out.t() if layout == "map" else out
    lists = torch.full((k, M, 3), 9.0, device="cuda")
    lists[:, :, 1] = top.t()
    places = torch.full((M, 2 * k), 1, dtype=torch.int32, device="cuda")
    places[:, ::2] = ids
    losses, g = dss.distill(z, lists[:, :, 1].t(), places[:, ::2], grad=grad)
    assert g is grad
    _check(losses, grad, z, top, ids)
    out.fill_(-77)
    assert bool((gb == -77).all())


def test_broadcast_operands():
    """One row of logits, one list, for all positions."""
    z, top, ids = _inputs(1, 50, 6)
    M = 40
    losses, grad = dss.distill(z.expand(M, 50), top.expand(M, 6), ids.expand(M, 6))
    _check(losses, grad, z.expand(M, 50), top.expand(M, 6), ids.expand(M, 6))


def test_offsets_over_32_bits():
    import torch
    far, M, C, k = 1 << 30, 6, 70, 5
    z, top, ids = _inputs(M, C, k, dtype="bf16")
    zb = torch.empty(6 * far, dtype=torch.bfloat16, device="cuda")
    gb = torch.empty(6 * far, dtype=torch.bfloat16, device="cuda")
    for shape, stride in (((M, C), (far, 1)), ((M, C), (1, far // 12))):
        zf, gf = zb.as_strided(shape, stride), gb.as_strided(shape, stride)
        zf.copy_(z)
        losses, _ = dss.distill(zf, top, ids, grad=gf)
        _check(losses, gf, z, top, ids)


@pytest.mark.parametrize("spread", [0.0, 30.0, 1000.0, 1e30])
def test_logits_of_any_size(spread):
    z, top, ids = _inputs(50, 40, 6, spread=spread)
    losses, grad = dss.distill(z, top, ids)
    _check(losses, grad, z, top, ids)


def test_gradient_is_the_losses_difference():
    """A step along the gradient changes the loss by its length: differences of the kernel's own losses."""
    import torch
    for layout in ("rows", "map"):
        z, top, ids = _inputs(200, 30, 6, layout, spread=1.0)
        _, grad = dss.distill(z, top, ids, temperature=2.0)
        h = 2.0 ** -6
        d = torch.randn(200, 30, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").sign()
        up, down = ((z + s * h * d) for s in (1, -1))
        a, b = (dss.distill(x, top, ids, temperature=2.0, with_grad=False)[0].double() for x in (up, down))
        # the third derivative of log sum exp along signs is at most 2 T^2 / T^3 = 1; the losses round by 2^-24 of some 40
        off = (a - b) / (2 * h) - (grad.double() * d.double()).sum(dim=1)
        assert float(off.abs().max()) < h * h / 6 * 8 + 40 * 2.0 ** -23 / h


def test_no_positions():
    import torch
    z = torch.empty((0, 8), device="cuda")
    losses, grad = dss.distill(z, torch.empty((0, 3), device="cuda"), torch.empty((0, 3), dtype=torch.int64, device="cuda"))
    assert losses.shape == (0,) and grad.shape == (0, 8)


def test_other_stream():
    import torch
    side = torch.cuda.Stream()
    for M, C in ((100, 40), (3, 50000), (3, 140000)):
        z, top, ids = _inputs(M, C, 7)
        ref = dss.distill(z, top, ids)
        side.wait_stream(torch.cuda.current_stream())
        got = dss.distill(z, top, ids, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(1, 4, 2), (300, 64, 8), (70, 700, 9), (3, 100000, 40)])
def test_graph_replays(M, C, k, layout):
    """Two captured calls that share a workspace, replayed in turn with new inputs."""
    import torch
    z, top, ids = _inputs(M, C, k, layout)
    room = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    outs = [(torch.empty(M, device="cuda"), torch.empty_like(z)) for _ in range(2)]
    graphs = []
    for n, (losses, grad) in enumerate(outs):
        call = lambda: dss.distill(z, top, ids, temperature=1.0 + n, losses=losses, grad=grad, workspace=room)  # noqa: E731
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for n in range(3):
        z.copy_(_inputs(M, C, k, layout, seed=n + 5)[0])
        room.fill_(255)
        for losses, grad in outs:
            losses.fill_(-3)
            grad.fill_(-3)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for i, (losses, grad) in enumerate(outs):
            want = dss.distill(z, top, ids, temperature=1.0 + i)
            assert torch.equal(losses, want[0]) and torch.equal(grad, want[1])


def test_binding_refusals():
    import torch
    z, top, ids = _inputs(6, 10, 3)
    w = torch.ones(6, device="cuda")
    bad = [lambda: dss.distill(z.half(), top, ids), lambda: dss.distill(z.cpu(), top, ids), lambda: dss.distill(z[0], top, ids),
           lambda: dss.distill(z, top[:5], ids), lambda: dss.distill(z, top, ids[:5]), lambda: dss.distill(z, top, ids[:, :2]),
           lambda: dss.distill(z, top[:, :0], ids[:, :0]), lambda: dss.distill(z, top, ids.float()),
           lambda: dss.distill(z, top.double(), ids), lambda: dss.distill(z, top.cpu(), ids),
           lambda: dss.distill(z, top, ids, weights=w[:5]), lambda: dss.distill(z, top, ids, weights=w.double()),
           lambda: dss.distill(z, top, ids, losses=w[:5]), lambda: dss.distill(z, top, ids, grad=z.bfloat16()),
           lambda: dss.distill(z, top, ids, grad=z, with_grad=False), lambda: dss.distill(z, top, ids, grad=z[:5]),
           lambda: dss.distill(z, top, ids, workspace=torch.empty(65536, dtype=torch.uint8))]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted", n)
    for call, status in ((lambda: dss.distill(z, top, ids, temperature=0.0), 1),
                         (lambda: dss.distill(z, top, ids, temperature=float("nan")), 1),
                         (lambda: dss.distill(z, top, ids, scale=float("inf")), 1),
                         (lambda: dss.distill(z, top, ids, grad=torch.empty((10, 6), device="cuda").t()), 1),
                         (lambda: dss.distill(z[:1].expand(6, 10), top, ids, grad=z[:1].expand(6, 10)), 1),
                         (lambda: dss.distill(z[::2, ::2], top[::2], ids[::2]), 3),
                         (lambda: dss.distill(*_inputs(2, 40000, 3), workspace=torch.empty(100, dtype=torch.uint8, device="cuda")), 2)):
        with pytest.raises(dss.DssError) as e:
            call()
        assert e.value.status == status
