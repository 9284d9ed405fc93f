"""8-bit tokens at the ends of their ranges: the most channels, the most tokens, and the parts of the products that
ordinary sizes do not reach.  Bounds as in test_gpu_tokens.py."""
import numpy as np
import pytest

from oracle import tokens
from paper_1508_06904_amd import dss
from tests.test_gpu_tokens import _check_layer
from tests.test_tile_choice import SHAPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------- channels up to 2^31 - 1

@pytest.mark.parametrize("M,K,dtype", [(1, 2 ** 31 - 1, "f32"), (1, 2 ** 31 - 256, "f32"), (2, 2 ** 31 - 1, "bf16"),
                                       (64, 2 ** 31 - 1, "f32")])
def test_channels_up_to_the_largest_count(M, K, dtype):
    """A token's value repeated over all of its channels (a stride of 0): every code is 127 or -127."""
    import torch
    if torch.cuda.mem_get_info()[0] < 1.2 * M * K:
        pytest.skip("the codes do not fit the free memory")
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    values = torch.linspace(-3, 5, M).add(0.125).to("cuda").to(dt)
    codes = torch.full((M, K), 55, dtype=torch.int8, device="cuda")
    _, scales = dss.quantize_tokens(values[:, None].expand(M, K), codes=codes)
    want, wsc = tokens.quantize(values[:, None].float().cpu().numpy())
    assert np.array_equal(scales.cpu().numpy(), wsc)
    want = torch.from_numpy(want).to("cuda")
    for k in range(0, K, 1 << 27):
        assert bool((codes[:, k:k + (1 << 27)] == want).all()), k


# ---------------------------------------------------------------------------- products

def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _weights(N, K, seed=0):
    rng = np.random.default_rng([seed, N, K, 1])
    return (_dev(rng.integers(-127, 128, (N, K)).astype(np.int8)), _dev((rng.random(N) * 0.02).astype(np.float32)),
            _dev(rng.standard_normal(N).astype(np.float32)))


@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("K,dtype", [(896, "f32"), (897, "f32"), (930, "f32"), (960, "f32"), (961, "f32"), (930, "bf16")])
def test_layers_of_maps_around_64_kb_of_lds(K, dtype, planar):
    """Coded and multiplied in one launch, the same bits as in two: binary32 tokens of 897 to 960 channels need
    just over 64 KB of LDS with the room for the largest values."""
    import torch
    M, N = 4200, 40
    gen = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn((K, M), generator=gen, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16).t()
    w, ws, bias = _weights(N, K)
    got = dss.linear_i8(x, w, ws, bias=bias, act="relu", planar=planar)
    assert torch.equal(got, dss.matmul_i8(*dss.quantize_tokens(x), w, ws, bias=bias, act="relu", planar=planar))


@pytest.mark.parametrize("planar", [False, True])
def test_an_output_of_another_type_than_asked_for_is_refused(planar):
    import torch
    M, N, K = 5, 3, 8
    x = torch.randn((M, K), device="cuda")
    w, ws, _ = _weights(N, K)
    q, s = dss.quantize_tokens(x)
    for have, ask in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float16)):
        out = torch.empty((N, M) if planar else (M, N), dtype=have, device="cuda")
        for call in (lambda **kw: dss.linear_i8(x, w, ws, **kw), lambda **kw: dss.matmul_i8(q, s, w, ws, **kw)):
            with pytest.raises(ValueError):
                call(out=out, out_dtype=ask, planar=planar)
            want = call(out_dtype=have, planar=planar)
            assert torch.equal(call(out=out, out_dtype=have, planar=planar), want)
            assert torch.equal(call(out=out, planar=planar), want)


@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("out,act", [("f32", "none"), ("f32", "relu"), ("bf16", "none"), ("bf16", "tanh")])
@pytest.mark.parametrize("tile,M,N,K", [(t,) + s for t in SHAPES for s in SHAPES[t]])
def test_every_tile(tile, M, N, K, out, act, planar):
    """Whole products on each of the four tiles, over several steps, with sides that no tile divides."""
    import torch
    rng = np.random.default_rng([M, N, K])
    codes, scales = rng.integers(-127, 128, (M, K)).astype(np.int8), (rng.random(M) * 0.02 + 1e-3).astype(np.float32)
    w, ws, bias = (t.cpu().numpy() for t in _weights(N, K))
    y = dss.matmul_i8(*map(_dev, (codes, scales, w, ws)), bias=_dev(bias), act=act, planar=planar,
                      out_dtype=torch.float32 if out == "f32" else torch.bfloat16)
    _check_layer(y.t() if planar else y, codes, scales, w, ws, bias, act, out == "bf16")


@pytest.mark.parametrize("M,N,K", [(20, 70_001, 77), (32, 8192, 130), (3, 20_000, 700), (13, 8400, 512), (32, 8193, 128),
                                   (1, 66_000, 96)])
def test_few_tokens_of_wide_layers(M, N, K):
    """More outputs than a launch's workgroups take at once, and either side of the streaming kernel's width."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn((M, K), generator=gen, device="cuda")
    w, ws, bias = _weights(N, K)
    q, s = dss.quantize_tokens(x)
    for planar in (False, True):
        y = dss.linear_i8(x, w, ws, bias=bias, planar=planar)
        assert torch.equal(y, dss.matmul_i8(q, s, w, ws, bias=bias, planar=planar))
        _check_layer(y.t() if planar else y, *(t.cpu().numpy() for t in (q, s, w, ws, bias)), "none")


@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("M,N,K,out", [(40_064, 512, 200, "f32"), (40_064, 1024, 130, "bf16"), (300_032, 64, 256, "f32")])
def test_large_outputs_of_whole_lines(M, N, K, out, planar):
    """Outputs of more than 64 MB whose rows are whole 128-byte lines are stored around the caches: the same bits as
    through them (one line's room more for each row), and nothing beside them."""
    import torch
    dt = torch.float32 if out == "f32" else torch.bfloat16
    rows, cols = (N, M) if planar else (M, N)
    assert rows * cols * dt.itemsize > 1 << 26 and cols * dt.itemsize % 128 == 0
    x = torch.randn((K, M) if planar else (M, K), generator=torch.Generator(device="cuda").manual_seed(K), device="cuda")
    x = x.t() if planar else x
    w, ws, bias = _weights(N, K)
    y = torch.full((rows, cols), -77.0, dtype=dt, device="cuda")
    assert y.data_ptr() % 128 == 0
    dss.linear_i8(x, w, ws, bias=bias, out=y, planar=planar)
    odd = torch.full((rows, cols + 1), -77.0, dtype=dt, device="cuda")
    dss.linear_i8(x, w, ws, bias=bias, out=odd[:, :cols], planar=planar)
    assert torch.equal(y, odd[:, :cols]) and bool((odd[:, cols] == -77).all())
    at = torch.randperm(M, generator=torch.Generator().manual_seed(1))[:2000].to("cuda")
    q, s = tokens.quantize(x[at].cpu().numpy())
    part = y[:, at].t() if planar else y[at]
    _check_layer(part, q, s, *(t.cpu().numpy() for t in (w, ws, bias)), "none", out == "bf16")


@pytest.mark.parametrize("planar", [False, True])
def test_copied_codes_in_two_parts(planar):
    """Rows of codes at odd addresses are copied 64 MB at a time: more of them than that, with copied weights."""
    import torch
    M, N, K = 70_001, 50, 1000
    assert M * 1008 > 1 << 26
    gen = torch.Generator(device="cuda").manual_seed(5)
    buf = torch.randint(-127, 128, (M, K + 3), generator=gen, device="cuda", dtype=torch.int8)
    scales = torch.rand(M, generator=gen, device="cuda") + 0.1
    w, ws, bias = _weights(N, K)
    y = dss.matmul_i8(buf[:, 3:], scales, w, ws, bias=bias, planar=planar)
    y = y.t() if planar else y
    for m in range(0, M, 10_000):
        part = slice(m, min(m + 10_000, M))
        _check_layer(y[part], *(t.cpu().numpy() for t in (buf[part, 3:], scales[part], w, ws, bias)), "none")


@pytest.mark.parametrize("planar", [False, True])
def test_more_tokens_than_a_launch_has(planar):
    """2^27 tokens and some: the second launch has shifted codes, scales and outputs, and the weights copied for
    the first (they lie at an odd address)."""
    import torch
    M, N, K = (1 << 27) + 1003, 3, 16
    gen = torch.Generator(device="cuda").manual_seed(6)
    codes = torch.randint(-127, 128, (M, K), generator=gen, device="cuda", dtype=torch.int8)
    scales = torch.rand(M, generator=gen, device="cuda") + 0.1
    w, ws, bias = _weights(N, K)
    odd = torch.zeros((N, K + 5), dtype=torch.int8, device="cuda")
    odd[:, 3:3 + K] = w
    y = dss.matmul_i8(codes, scales, odd[:, 3:3 + K], ws, bias=bias, out_dtype=torch.bfloat16, planar=planar)
    y = y.t() if planar else y
    at = torch.cat([torch.randint(0, M, (5000,), generator=torch.Generator().manual_seed(1)),
                    torch.arange((1 << 27) - 70, M)]).to("cuda")
    _check_layer(y[at], *(t.cpu().numpy() for t in (codes[at], scales[at], w, ws, bias)), "none", True)


@pytest.mark.parametrize("planar", [False, True])
def test_more_tokens_of_a_map_than_a_launch_codes(planar):
    """Over 2^21 tokens, coded and multiplied in one launch for each half, and the same bits as coded first."""
    import torch
    M, N, K = (1 << 21) + 71, 16, 256
    x = torch.randn((K, M), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda").t()
    w, ws, bias = _weights(N, K)
    y = dss.linear_i8(x, w, ws, bias=bias, planar=planar)
    assert torch.equal(y, dss.matmul_i8(*dss.quantize_tokens(x), w, ws, bias=bias, planar=planar))
    y = y.t() if planar else y
    half = (M + 1) // 2
    at = torch.cat([torch.arange(0, 70), torch.arange(half - 70, half + 70), torch.arange(M - 70, M)]).to("cuda")
    q, s = tokens.quantize(x[at].cpu().numpy())
    _check_layer(y[at], q, s, *(t.cpu().numpy() for t in (w, ws, bias)), "none")


def test_counts_that_the_library_does_not_take_are_refused():
    """Channels and outputs of 2^32 and some, which 32 bits would cut to those few."""
    import torch
    far = 2 ** 32
    x = torch.ones((1, 1), device="cuda").expand(1, far + 8)
    with pytest.raises(ValueError):
        dss.quantize_tokens(x)
    w, ws, _ = _weights(3, 8)
    for call in (lambda: dss.linear_i8(x, w, ws), lambda: dss.linear_i8(x[:, :2 ** 31], w, ws),
                 lambda: dss.linear_i8(x[:, :1], torch.empty((far + 3, 1), dtype=torch.int8, device="cuda"), ws),
                 lambda: dss.matmul_i8(torch.empty((1, far + 8), dtype=torch.int8, device="cuda"), ws[:1], w, ws),
                 lambda: dss.matmul_i8(w[:1, :1], ws[:1], torch.empty((far + 3, 1), dtype=torch.int8, device="cuda"), ws)):
        with pytest.raises(ValueError):
            call()


def test_a_stream_of_another_device_is_refused():
    """The tensors are checked to be on the current device; the kernels have to run there."""
    import types

    import torch
    here = torch.cuda.current_device()
    other = types.SimpleNamespace(device=torch.device("cuda", here + 1), cuda_stream=0)
    x = torch.randn((5, 8), device="cuda")
    w, ws, _ = _weights(3, 8)
    q, s = dss.quantize_tokens(x)
    for call in (lambda **kw: dss.quantize_tokens(x, codes=q, scales=s, **kw), lambda **kw: dss.linear_i8(x, w, ws, out=y, **kw),
                 lambda **kw: dss.matmul_i8(q, s, w, ws, out=y, **kw),
                 lambda **kw: dss.grad_norm([x], norm=norm, workspace=room, **kw),
                 lambda **kw: dss.clip_grads([x], 0.5, out=[z], norm=norm, workspace=room, **kw)):
        y, z, norm = torch.empty((5, 3), device="cuda"), torch.empty_like(x), torch.empty((), device="cuda")
        room = torch.empty(8192, dtype=torch.uint8, device="cuda")
        with pytest.raises(ValueError):
            call(stream=other)
        for stream in (torch.cuda.Stream(), torch.cuda.current_stream(), torch.cuda.default_stream()):
            stream.wait_stream(torch.cuda.current_stream())
            call(stream=stream)
            torch.cuda.current_stream().wait_stream(stream)
