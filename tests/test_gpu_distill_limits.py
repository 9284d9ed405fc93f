"""Distillation at the ends of its ranges: calls of several launches, the longest rows, the kernels' borders.  Bounds as in
test_gpu_distill.py."""
import pytest

from paper_1508_06904_amd import dss
from tests.test_gpu_distill import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _large(M, C, k, layout, dtype, seed=0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = (lambda n: (n, M)) if layout == "map" else (lambda n: (M, n))
    turn = (lambda t: t.t()) if layout == "map" else (lambda t: t)
    z = turn(torch.randn(shape(C), generator=gen, device="cuda", dtype=torch.float32 if dtype == "f32" else torch.bfloat16))
    top = turn(torch.randn(shape(k), generator=gen, device="cuda"))
    ids = turn(torch.randint(-1, C, shape(k), generator=gen, device="cuda", dtype=torch.int32))
    return z, top, ids


@pytest.mark.parametrize("M,C,k,layout,dtype", [
    ((1 << 21) + 700, 3, 2, "rows", "f32"),            # rows: two launches of four lanes for a row
    ((1 << 21) + 701, 130, 3, "map", "bf16"),          # tiles: two launches, the second one's last tile not whole
    (1 << 21, 140, 2, "map", "f32"),                 # tiles: a launch's very end
    (40_003, 1100, 5, "map", "bf16"),                  # parts: two slabs of positions
    (33_000, 1025, 70, "map", "f32"),
    (4_200, 66_000, 9, "rows", "f32"),                 # long rows: two launches
])
def test_calls_of_several_launches(M, C, k, layout, dtype):
    import torch
    z, top, ids = _large(M, C, k, layout, dtype)
    losses, grad = dss.distill(z, top, ids, temperature=2.0)
    at = torch.cat([torch.arange(60), torch.randint(0, M, (300,), generator=torch.Generator().manual_seed(1)),
                    torch.arange(M - 150, M)])
    at = torch.cat([at] + [torch.arange(border - 20, min(border + 20, M)) for border in (4096, 32768, (1 << 21) - 64, 1 << 21)
                           if border < M])
    at = at[:400].to("cuda") if C > 10_000 else at.to("cuda")
    _check(losses[at], grad[at], z[at], top[at], ids[at], T=2.0)
    alone, none = dss.distill(z, top, ids, temperature=2.0, with_grad=False)
    _check(alone[at], None, z[at], top[at], ids[at], T=2.0)


# the borders between the kernels: threads for a row, columns, tiles, parts, workgroups that share a position
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(70, c, k) for c in (63, 64, 65, 127, 128, 129, 255, 256, 257, 512, 513, 1023, 1024, 1025)
                                   for k in (1, 8, 9)] +
                         [(5, c, 20) for c in (2048, 2049, 4096, 4097, 8192, 8193, 16383, 16384, 16385, 32768, 32769, 65536,
                                               65537, 131072, 131073)] + [(130, 65537, 3), (127, 65537, 3), (130, 16384, 3), (200, 300, 128), (200, 300, 129),
                                                          (31, 200, 4), (32, 200, 4), (63, 200, 4), (64, 200, 4)])
def test_kernels_borders(M, C, k, layout, dtype):
    z, top, ids = _inputs(M, C, min(k, C), layout, dtype, repeat=k > 100)
    losses, grad = dss.distill(z, top, ids, scale=3.0)
    _check(losses, grad, z, top, ids, scale=3.0)


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(3, 140, 128), (70, 130, 128), (66, 1500, 128), (40, 200, 200), (20, 2000, 1024), (65, 90, 1024)])
def test_long_lists_of_one_class(M, C, k, layout):
    """All places of a list have one class, or take turns with another."""
    z, top, ids = _inputs(M, C, min(k, C), layout)
    top, ids = (t[:, :1].expand(M, k).contiguous() for t in (top, ids.clamp(min=0)))
    ids[:, 1::2] = (ids[:, 1::2] + 1) % C
    ids[0] = ids[0, 0]
    losses, grad = dss.distill(z, top, ids)
    _check(losses, grad, z, top, ids)


@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,C,k", [(70, 64, 8), (70, 500, 8), (70, 2000, 8), (9, 40000, 8), (9, 70000, 8), (130, 600, 130),
                                   (16384, 1100, 8), (32768, 1300, 40)])
def test_the_same_call_gives_the_same_bits(M, C, k, layout):
    import torch
    z, top, ids = _inputs(M, C, k, layout, repeat=True)
    first = dss.distill(z, top, ids)
    for _ in range(5):
        again = dss.distill(z, top, ids)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_two_streams_with_workspaces_of_their_own():
    import torch
    sides = [torch.cuda.Stream() for _ in range(2)]
    cases = [_inputs(40, 70000, 9, "rows", seed=1), _inputs(50, 3000, 9, "map", seed=2)]
    want = [dss.distill(*c) for c in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for n, (side, c) in enumerate(zip(sides, cases)):
            got[n].append(dss.distill(*c, stream=side))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w[0], a) and torch.equal(w[1], b) for a, b in g)


def test_largest_and_smallest_temperatures():
    import torch
    for layout in ("rows", "map"):
        for C in (20, 300, 3000):
            z, top, ids = _inputs(40, C, 5, layout)
            for T in (2.0 ** -60, 2.0 ** 60, 1e-3, 1e3):
                # of its own size, so that only the temperature is extreme
                zs, ts = z * T, top * T
                scale = 2.0 ** -40 if T > 1e10 else 1.0
                losses, grad = dss.distill(zs, ts, ids, temperature=T, scale=scale)
                _check(losses, grad, zs, ts, ids, T=T, scale=scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,layout", [(9000, 4100, "rows"), (4400, 9000, "rows"), (1200, 33000, "rows"), (700, 70_001, "rows"),
                                        (600, 140_000, "rows"), (1 << 20, 40, "map"), (1 << 18, 200, "map"), (32768, 1100, "map"),
                                        (70_016, 1030, "map"), ((1 << 20) + 3, 40, "map")])
def test_calls_around_the_caches(M, C, layout, dtype):
    """Calls too large for the caches, over their logits too, write nothing else; where one workgroup has all of a position they
    give the bits of calls that fit the caches."""
    import torch
    z, top, ids = _large(M, C, 4, layout, dtype)
    assert M * C * z.element_size() > 1 << 26
    losses, grad = dss.distill(z, top, ids, temperature=0.5)
    few = (1 << 26) // (C * z.element_size()) // 64 * 64
    alone = C < 1024 if layout == "map" else C < 65536
    for at in (0, M // 128 * 64, M - few):
        part = slice(at, at + few)
        if alone:
            some, grads = dss.distill(z[part], top[part], ids[part], temperature=0.5)
            assert torch.equal(some, losses[part]) and torch.equal(grads, grad[part])
        part = slice(at, at + min(few, 64))
        _check(losses[part], grad[part], z[part], top[part], ids[part], T=0.5)
    only, _ = dss.distill(z, top, ids, temperature=0.5, with_grad=False)
    _check(only[part], None, z[part], top[part], ids[part], T=0.5)
    rows, cols = (C, M) if layout == "map" else (M, C)
    buf = torch.full((rows + 2, cols + 64), -77.0, dtype=z.dtype, device="cuda")
    over = buf[1:rows + 1, 64:]
    over.copy_(z.t() if layout == "map" else z)
    over = over.t() if layout == "map" else over
    again, _ = dss.distill(over, top, ids, temperature=0.5, grad=over)
    assert torch.equal(again, losses) and torch.equal(over, grad)
    over.fill_(-77)
    assert bool((buf == -77).all())
