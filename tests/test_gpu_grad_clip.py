"""The gradient norm and clipping against the oracle's 64-bit form.

Tolerances.  The norm is a binary64 sum of exact squares (n terms: relative error below n 2^-53,
under 2^-30 for every size here) rounded to binary32: 2^-24, 1.01 of it with the rest.  A clipped
value is the factor rounded to binary32 and a binary32 product, 2 * 2^-24 of the value and, near the
smallest numbers, half of the smallest one; in bfloat16 a last rounding to 8 bits, 2^-8 more."""
import numpy as np
import pytest

from oracle import tokens
from paper_1508_06904_amd import dss, workloads as wl

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()


def _np(t):
    return t.detach().float().cpu().numpy()


def _check_norm(norm, want):
    got = float(norm)
    assert abs(got - want) <= 1.01 * U * want, (got, want)


def _check_clipped(got, grad, want):
    import torch
    rel = 2.02 * U + (2.0 ** -8 if grad.dtype == torch.bfloat16 else 0)
    small = 2.0 ** -134 if grad.dtype == torch.bfloat16 else 2.0 ** -149
    assert got.shape == grad.shape and got.dtype == grad.dtype
    assert np.all(np.abs(_np(got) - want) <= rel * np.abs(want) + small)


def _grads(sizes, seed=0, dtype="f32", scale=1.0):
    import torch
    rng = np.random.default_rng(seed)
    dt = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.float32, torch.bfloat16]}[dtype]
    return [torch.from_numpy((rng.standard_normal(s) * scale).astype(np.float32)).to("cuda").to(dt[n % len(dt)])
            for n, s in enumerate(sizes)]


SIZES = {
    "one": [1], "empty_list": [], "empty_tensors": [0, 0], "with_empty": [0, 5, 0, 4097, 0],
    "vector_edges": [3, 4, 5, 7, 8, 9, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 16384, 16385],
    "large": [(1 << 22) + 13], "over_the_runs": [40_000_003, 17],
    "a_table": [33] * 112, "a_table_and_one": [33] * 113, "tables": list(range(1, 400)),
    "network": [(64, 3, 5, 5), 64, (128, 64, 5, 5), 128, (2, 512, 1, 1), 2],
}


@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("name", SIZES)
def test_norm_and_clipping(name, dtype):
    import torch
    grads = _grads(SIZES[name], seed=len(name), dtype=dtype)
    before = [g.clone() for g in grads]
    want = tokens.grad_norm([_np(g) for g in grads])
    _check_norm(dss.grad_norm(grads), want)
    for bound in (0.25 * want, 2 * want + 1, 0.0, float("inf")):
        norm, out = dss.clip_grads(grads, bound)
        _check_norm(norm, want)
        ref = tokens.clip([_np(g) for g in grads], np.float32(bound))[1]
        for o, g, r in zip(out, grads, ref):
            _check_clipped(o, g, r)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    norm, out = dss.clip_grads(grads, 0.25 * want, out=grads)       # in place: the same bits
    ref = dss.clip_grads(before, 0.25 * want)[1]
    assert all(o is g for o, g in zip(out, grads))
    assert all(torch.equal(a, b) for a, b in zip(grads, ref))


def test_below_the_bound_nothing_changes_in_place():
    import torch
    grads = _grads([100_001, 7], seed=3)
    before = [g.clone() for g in grads]
    dss.clip_grads(grads, 1e6, out=grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e19, 1e30])
def test_squares_outside_binary32(scale):
    """Squares that binary32 would lose (below 2^-149) or call infinite (above 2^128)."""
    grads = _grads([5000, 333], seed=5, scale=scale)
    norm, out = dss.clip_grads(grads, 1.0)
    want, ref = tokens.clip([_np(g) for g in grads], 1.0)
    _check_norm(norm, want)
    for o, g, r in zip(out, grads, ref):
        _check_clipped(o, g, r)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 4098, 20_000])
def test_values_that_are_no_numbers(bad, at):
    grads = _grads([20_001, 9], seed=6)
    grads[0][at] = bad
    norm, out = dss.clip_grads(grads, 1.0)
    want, ref = tokens.clip([_np(g) for g in grads], 1.0)
    assert np.array_equal(np.float64(float(norm)), np.float64(want), equal_nan=True)
    assert float(dss.grad_norm(grads)) == float(norm) or np.isnan(want)
    for o, r in zip(out, ref):
        assert np.array_equal(np.isnan(_np(o)), np.isnan(r)) and np.all(_np(o)[~np.isnan(r)] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_at_any_element_and_nothing_beside_them(dtype):
    """Tensors of all alignments in one buffer, inputs and outputs aligned differently; what
    lies between the outputs stays."""
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    src = torch.randn(60_000, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dt)
    dst = torch.full((70_000,), -77.0, dtype=dt, device="cuda")
    grads, outs, at, to = [], [], 0, 3
    keep = torch.ones(70_000, dtype=torch.bool, device="cuda")
    for n in (1, 2, 3, 5, 1021, 4099, 8191, 4096, 12_345, 9_999):
        grads.append(src[at:at + n])
        outs.append(dst[to:to + n])
        keep[to:to + n] = False
        at += n + 1
        to += n + 3
    norm, _ = dss.clip_grads(grads, 1.0, out=outs)
    want, ref = tokens.clip([_np(g) for g in grads], 1.0)
    _check_norm(norm, want)
    for o, g, r in zip(outs, grads, ref):
        _check_clipped(o, g, r)
    assert bool((dst[keep] == -77).all())


def test_other_orders_of_the_axes():
    import torch
    a = _grads([(6, 5, 4, 3)], seed=8)[0]
    g = [a.permute(0, 2, 3, 1).contiguous().permute(0, 3, 1, 2), a.t() if a.dim() == 2 else a[0, 0].t()]
    assert not g[0].is_contiguous() and not g[1].is_contiguous()
    norm, out = dss.clip_grads(g, 0.5)
    want, ref = tokens.clip([_np(t) for t in g], 0.5)
    _check_norm(norm, want)
    for o, t, r in zip(out, g, ref):
        _check_clipped(o, t, r)


def test_lists_of_more_values_than_the_caches_hold():
    """Over 2^28 values, in bfloat16: the way around the caches, with the oracle's sums in 64 bits on the GPU."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    grads = [torch.randn(n, generator=gen, device="cuda", dtype=torch.bfloat16) for n in ((1 << 28) - 7, 100_003, 5)]
    want = float(torch.sqrt(sum((g.double() ** 2).sum() for g in grads)))
    _check_norm(dss.grad_norm(grads), want)
    norm, out = dss.clip_grads(grads, 1.0)
    _check_norm(norm, want)
    for o, g in zip(out, grads):
        ref = g.double() * (1.0 / (want + 1e-6))
        assert bool(((o.double() - ref).abs() <= (2.02 * U + 2.0 ** -8) * ref.abs() + 2.0 ** -134).all())


def test_same_gradients_same_bits():
    import torch
    grads = _grads([1_000_003, 77, 300_000], seed=9)
    first = dss.clip_grads(grads, 0.1)
    for _ in range(3):
        again = dss.clip_grads(grads, 0.1)
        assert torch.equal(first[0], again[0]) and all(torch.equal(a, b) for a, b in zip(first[1], again[1]))


def test_other_stream():
    import torch
    side = torch.cuda.Stream()
    grads = _grads([500_000, 1001], seed=10)
    ref = dss.clip_grads(grads, 0.3)
    side.wait_stream(torch.cuda.current_stream())
    got = dss.clip_grads(grads, 0.3, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(ref[0], got[0]) and all(torch.equal(a, b) for a, b in zip(ref[1], got[1]))


def test_graph_replays():
    import torch
    grads = _grads([70_000, 33, 4097], seed=11)
    out = [torch.empty_like(g) for g in grads]
    norm = torch.empty((), device="cuda")
    ws = torch.empty(dss.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    dss.clip_grads(grads, 0.7, out=out, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dss.clip_grads(grads, 0.7, out=out, norm=norm, workspace=ws)
    for n in range(3):
        for g, new in zip(grads, _grads([70_000, 33, 4097], seed=20 + n)):
            g.copy_(new)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        ref = dss.clip_grads(grads, 0.7)
        assert torch.equal(norm, ref[0]) and all(torch.equal(a, b) for a, b in zip(out, ref[1]))


def test_gradients_of_a_network():
    """The flat gradients of a backward pass and their per-convolution views have one norm."""
    import torch
    w = wl.make("c3_512", H=76, W=81, widths=(16, 32, 48, 64))
    plan = dss.Plan.from_workload(w)
    x = torch.from_numpy(w.x).to("cuda")
    g = torch.ones_like(plan.eval_dense(x))
    gw, gb, _ = plan.backward(x, g, with_signal_grad=False)
    ws, bs = plan.split_grads(gw, gb)
    want, ref = tokens.clip([_np(t) for t in ws + bs], 1.0)
    _check_norm(dss.grad_norm([gw, gb]), want)
    norm, _ = dss.clip_grads(ws + bs, 1.0, out=ws + bs)
    _check_norm(norm, want)
    for t, r in zip(ws + bs, ref):
        _check_clipped(t, t, r)


def test_refusals():
    import torch
    g = _grads([(8, 6)], seed=1)[0]
    for bad in ([g.half()], [g.cpu()], [g[:, :3]], [g[::2]], [g.expand(2, 8, 6)], [g, 1.0], g):
        with pytest.raises(ValueError):
            dss.grad_norm(bad)
    for out in ([], [g.bfloat16()], [g.t()], [g, g], [torch.empty(6, 8, device="cuda").t()]):
        with pytest.raises(ValueError):
            dss.clip_grads([g], 1.0, out=out)
    for bound in (-1.0, float("nan")):
        with pytest.raises(dss.DssError) as e:
            dss.clip_grads([g], bound)
        assert e.value.status == 1
    with pytest.raises(dss.DssError):
        dss.grad_norm([g], workspace=torch.empty(4096, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        dss.grad_norm([g], norm=torch.empty(2, device="cuda"))
