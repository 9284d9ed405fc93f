"""Gradient clipping at the ends of its ranges: bounds and norms that are infinite, factors that binary32 cannot
hold with all of its bits, lists of every kernel."""
import numpy as np
import pytest

from oracle import tokens
from paper_1508_06904_amd import dss

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LISTS = {"one launch": [700, 0, 33], "runs": [70_000, 4097, 1], "tables": [300] * 130 + [9000]}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()


def _np(t):
    return t.detach().float().cpu().numpy()


def _grads(sizes, dtype, scale=1.0, seed=0):
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rng = np.random.default_rng(seed)
    return [torch.from_numpy((rng.standard_normal(s) * scale).astype(np.float32)).to("cuda").to(dt) for s in sizes]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), None])
@pytest.mark.parametrize("name", LISTS)
def test_an_infinite_bound_clips_nothing(name, bad, dtype, in_place):
    import torch
    grads = _grads(LISTS[name], dtype)
    if bad is not None:
        grads[-1][-1] = bad
    before = [g.clone() for g in grads]
    norm, out = dss.clip_grads(grads, float("inf"), out=grads if in_place else None)
    want, ref = tokens.clip([_np(g) for g in before], float("inf"))
    if bad is None:
        assert abs(float(norm) - want) <= 1.01 * U * want
    else:
        assert np.array_equal(np.float64(float(norm)), np.float64(want), equal_nan=True)
    for o, g, r in zip(out, before, ref):
        assert np.array_equal(_np(o), r, equal_nan=True)
        if bad != bad and g.numel():
            assert bool(torch.isnan(o).all())
        elif bad == bad:
            assert torch.equal(o, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,bound", [(1e5, 1e-35), (1e20, 1e-20), (1e25, 1e-25), (1e37, 1e-37), (1e37, 1e-44), (1e-3, 1e-42),
                                         (1e30, 1e-7), (1e3, 1e-36)])
@pytest.mark.parametrize("name", LISTS)
def test_factors_below_the_normal_numbers(name, scale, bound, dtype):
    """The factor bound / norm loses its bits in binary32 where the clipped values need not.  Rounding: the factor and
    the product 2 * 2^-24 of the value; near the smallest numbers the product is rounded once more, to half of
    the smallest one, and one of them covers that; bfloat16 as in every clipping."""
    grads = _grads(LISTS[name], dtype, scale)
    _, out = dss.clip_grads(grads, bound)
    ref = tokens.clip([_np(g) for g in grads], np.float32(bound))[1]
    rel = 2.02 * U + (2.0 ** -8 if dtype == "bf16" else 0)
    for o, r in zip(out, ref):
        assert np.all(np.abs(_np(o) - r) <= rel * np.abs(r) + (2.0 ** -133 if dtype == "bf16" else 2.0 ** -149))


def test_outputs_of_other_shapes_are_refused():
    """As many elements are not enough: a contiguous output of another shape would be filled in another order."""
    import torch
    grads = _grads([(8, 6), 5], "f32")
    make = lambda *shapes: [torch.full(s, -7.0, device="cuda") for s in shapes]  # noqa: E731
    for shapes in [((6, 8), (5,)), ((48,), (5,)), ((8, 6), (5, 1)), ((8, 6, 1), (5,)), ((5,), (8, 6)), ((8, 6),)]:
        out = make(*shapes)
        with pytest.raises(ValueError):
            dss.clip_grads(grads, 1.0, out=out)
        assert all(bool((o == -7).all()) for o in out)
    # other strides: refused unless all tensors are contiguous
    with pytest.raises(ValueError):
        dss.clip_grads([grads[0].t(), grads[1]], 1.0, out=make((6, 8), (5,)))
    out = make((8, 6), (5,))
    dss.clip_grads(grads, 1.0, out=out)
    dss.clip_grads([grads[0].t(), grads[1]], 1.0, out=[out[0].t(), out[1]])
    with pytest.raises(ValueError):
        dss.clip_grads([grads[0], 2.0], 1.0)
    with pytest.raises(ValueError):
        dss.clip_grads(grads, 1.0, out=[None, None])


def test_a_tensor_is_written_once():
    """Two entries of one list that write the same memory would race: scaled once, or twice.  Reading one twice is
    no matter, nor are any number of empty tensors."""
    import torch
    a, b, empty = _grads([5000, 40, 0], "f32")
    before = a.clone()
    for grads, out in (([a, a], "in place"), ([a, b, a], "in place"), ([a, a], [b.new_empty(5000)] * 2),
                       ([a, empty, a, empty], [a, empty, a, empty])):
        with pytest.raises(ValueError):
            dss.clip_grads(grads, 0.5, out=grads if out == "in place" else out)
        assert torch.equal(a, before)
    norm, out = dss.clip_grads([a, a, empty, empty], 0.5)
    want, ref = tokens.clip([_np(a), _np(a)], 0.5)
    assert abs(float(norm) - want) <= 1.01 * U * want and torch.equal(out[0], out[1])
    assert np.all(np.abs(_np(out[0]) - ref[0]) <= 2.02 * U * np.abs(ref[0]) + 2.0 ** -149)
    dss.clip_grads([empty, a, empty], 0.5, out=[empty, a, empty])


def test_binary32_lists_beyond_the_caches():
    """Over 2^28 values: loads and stores around the caches, against sums and products in 64 bits on the GPU."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    grads = [torch.randn(n, generator=gen, device="cuda") for n in ((1 << 28) - 7, 100_003, 5)]
    want = float(torch.sqrt(sum((g.double() ** 2).sum() for g in grads)))
    for bound in (1.0, 1e9):
        norm, out = dss.clip_grads(grads, bound)
        assert abs(float(norm) - want) <= 1.01 * U * want
        assert abs(float(dss.grad_norm(grads)) - want) <= 1.01 * U * want
        for o, g in zip(out, grads):
            ref = g.double() * min(1.0, bound / (want + 1e-6))
            assert bool(((o.double() - ref).abs() <= 2.02 * U * ref.abs() + 2.0 ** -149).all())
    before = [o.clone() for o in dss.clip_grads(grads, 1.0)[1]]
    dss.clip_grads(grads, 1.0, out=grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


def test_strides_that_do_not_matter():
    """Beside a tensor in another order of its axes: one of a single row out of a wider buffer, and empty ones, whose
    outputs have other strides for the same order of elements."""
    import torch
    wide = torch.randn((4, 100), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    grads = [wide[:, :6].contiguous().t(), wide.as_strided((1, 5), (100, 1)), wide[:, :0], wide[:0, 3:7]]
    want, ref = tokens.clip([_np(g) for g in grads], 0.5)
    outs = [torch.empty((4, 6), device="cuda").t()] + [torch.empty(g.shape, device="cuda") for g in grads[1:]]
    for out in (None, outs):
        norm, got = dss.clip_grads(grads, 0.5, out=out)
        assert abs(float(norm) - want) <= 1.01 * U * want
        for o, g, r in zip(got, grads, ref):
            assert o.shape == g.shape and np.all(np.abs(_np(o) - r) <= 2.02 * U * np.abs(r) + 2.0 ** -149)
    outs[0] = torch.empty((6, 4), device="cuda")
    with pytest.raises(ValueError):
        dss.clip_grads(grads, 0.5, out=outs)
