"""4-bit tokens at the ends of their ranges: the most channels, the most tokens, and the parts of the products that
ordinary sizes do not reach.  Bounds as in test_gpu_mx4.py."""
import types

import numpy as np
import pytest

from oracle import mx4
from paper_1508_06904_amd import dss
from tests.test_gpu_mx4 import _check_layer, _coded, _dev, _np, _x
from tests.test_mx4_tile_choice import SHAPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    dss.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------- codes

@pytest.mark.parametrize("M,K,layout", [(1, 2 ** 31 - 1, "rows"), (2, 2 ** 31 - 64, "rows"), (3, 2 ** 30 + 5, "map"),
                                        (70, 2 ** 26 + 9, "map")])
def test_channels_up_to_the_largest_count(M, K, layout):
    """A token's value repeated over all of its channels (a stride of 0): every code is 4 / 4, and its sign."""
    import torch
    B = -(-K // 32)
    values = torch.linspace(-3, 5, M).add(0.125).to("cuda")
    x = values[:, None].expand(M, K) if layout == "rows" else values[None].expand(K, M).t()
    codes = torch.full((M, 16 * B), 55, dtype=torch.uint8, device="cuda")
    _, scales = dss.quantize_mx4(x, codes=codes)
    want, wsc = map(_dev, mx4.quantize(np.repeat(values.cpu().numpy()[:, None], 32, axis=1)))
    assert bool((scales == wsc).all())
    whole = K // 32 * 16
    for k in range(0, whole, 1 << 26):
        part = codes[:, k:min(k + (1 << 26), whole)]
        assert bool((part.view(M, -1, 16) == want[:, None]).all()), k
    tail = torch.zeros((M, 16), dtype=torch.uint8, device="cuda")
    tail[:, :(K % 32) // 2] = want[:, :(K % 32) // 2]
    if K % 2:
        tail[:, (K % 32) // 2] = want[:, 0] & 15
    if K % 32:
        assert torch.equal(codes[:, whole:], tail)


@pytest.mark.parametrize("layout,K", [("rows", 1), ("rows", 33), ("map", 2), ("map", 33)])
def test_more_tokens_than_a_launch_codes(layout, K):
    """Over 2^28 tokens of few channels, sampled: codes and their values."""
    import torch
    M = (1 << 28) + 1001 if K < 3 else (1 << 27) + 1001
    gen = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn((K, M) if layout == "map" else (M, K), generator=gen, device="cuda", dtype=torch.bfloat16)
    x = x.t() if layout == "map" else x
    codes, scales = dss.quantize_mx4(x)
    at = torch.cat([torch.arange(300), torch.randint(0, M, (5000,), generator=torch.Generator().manual_seed(1)),
                    torch.arange(M - 1300, M)]).to("cuda")
    want, wsc = mx4.quantize(_np(x[at]))
    assert np.array_equal(codes[at].cpu().numpy(), want) and np.array_equal(scales[:, at].cpu().numpy(), wsc)
    del x
    v = dss.dequantize_mx4(codes, scales, K, out_dtype=torch.bfloat16, planar=layout == "map")
    v = v[:, at].t() if layout == "map" else v[at]
    assert np.array_equal(_np(v), mx4.values(want, wsc, K))


# ---------------------------------------------------------------------------- products

@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("out,act", [("f32", "none"), ("f32", "relu"), ("bf16", "none"), ("bf16", "tanh")])
@pytest.mark.parametrize("tile,M,N,K", [(t,) + s for t in SHAPES for s in SHAPES[t]])
def test_every_tile(tile, M, N, K, out, act, planar):
    """Whole products on each of the tiles, over several steps, with sides that no tile divides."""
    import torch
    tokens, weight = _coded(M, K, 7), _coded(N, K, 8)
    bias = np.random.default_rng(N).standard_normal(N).astype(np.float32)
    y = dss.matmul_mx4(*map(_dev, tokens + weight), bias=_dev(bias), act=act, planar=planar,
                       out_dtype=torch.float32 if out == "f32" else torch.bfloat16)
    _check_layer(y.t() if planar else y, mx4.values(*tokens), mx4.values(*weight), bias, act, out == "bf16")


@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("M,N,K", [(3, 40, 120_000), (16, 20, 100_000), (2, 35, 300_000), (16, 5, 260_001), (40, 3, 270_000),
                                   (1, 1, 1 << 20)])
def test_long_rows_on_one_side_few(M, N, K, planar):
    """Rows of which LDS holds fewer than there are, or none."""
    import torch
    tokens, weight = _coded(M, K, 9), _coded(N, K, 10)
    bias = np.random.default_rng(N).standard_normal(N).astype(np.float32)
    y = dss.matmul_mx4(*map(_dev, tokens + weight), bias=_dev(bias), planar=planar)
    _check_layer(y.t() if planar else y, mx4.values(*tokens), mx4.values(*weight), bias)


@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("M,N", [(40, 30), (50, 64)])
def test_rows_far_apart(M, N, planar):
    """Row strides over 8 MB, which the tiles do not take; offsets over 32 bits."""
    import torch
    K, far = 300, 1 << 27
    tokens, weight = _coded(M, K, 11), _coded(N, K, 12)
    wide = torch.empty((max(M, N) + 1) * far, dtype=torch.uint8, device="cuda")
    tc, wc = wide.as_strided((M, 160), (far, 1)), wide.as_strided((N, 160), (far, 1), 1024)
    tc.copy_(_dev(tokens[0]))
    wc.copy_(_dev(weight[0]))
    out = torch.empty(9 * (1 << 29) if min(M, N) <= 9 else 64 * far // 4, device="cuda", dtype=torch.bfloat16)
    ob = out.as_strided((N, M) if planar else (M, N), (far // 8, 1))
    dss.matmul_mx4(tc, _dev(tokens[1]), wc, _dev(weight[1]), out=ob, planar=planar)
    _check_layer(ob.t() if planar else ob, mx4.values(*tokens), mx4.values(*weight), None, "none", True)


@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("layout", ["rows", "map"])
@pytest.mark.parametrize("M,N,K,out", [(40_064, 512, 200, "f32"), (40_064, 1024, 130, "bf16"), (300_032, 64, 256, "f32"),
                                       (300_032, 120, 500, "f32")])
def test_large_outputs_of_whole_lines(M, N, K, out, layout, planar):
    """Outputs of more than 64 MB whose rows may be whole 128-byte lines are stored around the caches: the same bits as
    through them (one element's room more for each row), and nothing beside them."""
    import torch
    dt = torch.float32 if out == "f32" else torch.bfloat16
    rows, cols = (N, M) if planar else (M, N)
    assert rows * cols * dt.itemsize > 1 << 26
    x = _x(M, K, layout)
    w, ws = map(_dev, _coded(N, K, 13))
    y = torch.full((rows, cols), -77.0, dtype=dt, device="cuda")
    assert y.data_ptr() % 128 == 0
    dss.linear_mx4(x, w, ws, out=y, planar=planar)
    odd = torch.full((rows, cols + 1), -77.0, dtype=dt, device="cuda")
    dss.linear_mx4(x, w, ws, out=odd[:, :cols], planar=planar)
    assert torch.equal(y, odd[:, :cols]) and bool((odd[:, cols] == -77).all())
    at = torch.randperm(M, generator=torch.Generator().manual_seed(1))[:2000].to("cuda")
    part = y[:, at].t() if planar else y[at]
    _check_layer(part, mx4.values(*mx4.quantize(_np(x[at]))), mx4.values(w.cpu().numpy(), ws.cpu().numpy()), None, "none",
                 out == "bf16")


@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(256, 1, 2), (257, 64, 33), (511, 64, 256), (300, 17, 129), (32768, 200, 511), (32769, 33, 300),
                                   (33000, 256, 128), (40001, 250, 512), (35003, 400, 256)])
def test_layers_of_maps_in_one_launch(M, N, K, dtype, planar):
    """Coded and multiplied in one launch, into a buffer whose other elements stay; a block that is no number among the
    last tokens, which spoils that token alone, as in two calls."""
    import torch
    x = _x(M, K, "map", dtype).t().contiguous().t()
    x[M - 2, K // 2] = float("nan")
    weight = _coded(N, K, 14)
    bias = np.random.default_rng(N).standard_normal(N).astype(np.float32)
    rows, cols = (N, M) if planar else (M, N)
    buf = torch.full((rows + 2, cols + 5), -77.0, device="cuda")
    out = buf[1:rows + 1, 2:2 + cols]
    dss.linear_mx4(x, *map(_dev, weight), bias=_dev(bias), act="relu", out=out, planar=planar)
    y = out.t() if planar else out
    at = torch.cat([torch.arange(0, min(M, 700)), torch.arange(max(0, M - 700), M)]).unique().to("cuda")
    _check_layer(y[at], mx4.values(*mx4.quantize(_np(x[at]))), mx4.values(*weight), bias, "relu")
    two = dss.matmul_mx4(*dss.quantize_mx4(x), *map(_dev, weight), bias=_dev(bias), act="relu")
    assert torch.equal(torch.isnan(y), torch.isnan(two)) and int(torch.isnan(y).any(dim=1).sum()) == 1
    _check_layer(two[at], mx4.values(*mx4.quantize(_np(x[at]))), mx4.values(*weight), bias, "relu")
    out.fill_(-77)
    assert bool((buf == -77).all())


def test_many_tokens_of_a_map():
    """More outputs than 2^31, in one launch and from codes: a map of 17 million windows, sampled."""
    import torch
    M, K, N = 17_000_003, 40, 128
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((K, M), generator=gen, device="cuda").to(torch.bfloat16)
    weight = _coded(N, K, 15)
    w, ws = map(_dev, weight)
    at = torch.cat([torch.arange(5), torch.randint(0, M, (3000,), generator=torch.Generator().manual_seed(1)),
                    torch.arange(M - 70, M), torch.arange((1 << 21) - 9, (1 << 21) + 9)]).to("cuda")
    v = mx4.values(*mx4.quantize(_np(x[:, at].t())))
    y = dss.linear_mx4(x.t(), w, ws, out_dtype=torch.bfloat16, planar=True)
    _check_layer(y[:, at].t(), v, mx4.values(*weight), None, "none", True)
    codes, scales = dss.quantize_mx4(x.t())
    dss.matmul_mx4(codes, scales, w, ws, out=y, planar=True)
    _check_layer(y[:, at].t(), v, mx4.values(*weight), None, "none", True)


@pytest.mark.parametrize("planar", [False, True])
def test_more_tokens_than_a_launch_multiplies(planar):
    """2^27 tokens and some on tiles: the second launch has shifted codes, scales and outputs."""
    import torch
    M, N, K = (1 << 27) + 1003, 17, 20
    gen = torch.Generator(device="cuda").manual_seed(6)
    codes = torch.randint(0, 256, (M, 16), generator=gen, device="cuda", dtype=torch.uint8)
    codes[:, 10:] = 0
    scales = torch.randint(121, 130, (1, M), generator=gen, device="cuda", dtype=torch.uint8)
    weight = _coded(N, K, 16)
    bias = np.random.default_rng(N).standard_normal(N).astype(np.float32)
    y = dss.matmul_mx4(codes, scales, *map(_dev, weight), bias=_dev(bias), out_dtype=torch.bfloat16, planar=planar)
    y = y.t() if planar else y
    at = torch.cat([torch.randint(0, M, (5000,), generator=torch.Generator().manual_seed(1)),
                    torch.arange((1 << 27) - 70, M)]).to("cuda")
    _check_layer(y[at], mx4.values(codes[at].cpu().numpy(), scales[:, at].cpu().numpy()), mx4.values(*weight), bias, "none", True)


def test_counts_that_the_library_does_not_take_are_refused():
    """Channels, blocks and outputs of 2^31 and more, which 32 bits would cut to fewer."""
    import torch
    far = 2 ** 32
    x = torch.ones((1, 1), device="cuda").expand(1, far + 8)
    w, ws = map(_dev, _coded(3, 8))
    byte = torch.zeros((1, 1), dtype=torch.uint8, device="cuda")
    many = byte.expand(1, 16 * (2 ** 27)), byte.expand(2 ** 27, 1)
    for call in (lambda: dss.quantize_mx4(x), lambda: dss.linear_mx4(x, w, ws), lambda: dss.matmul_mx4(*many, *many),
                 lambda: dss.dequantize_mx4(*many),
                 lambda: dss.matmul_mx4(w[:1], ws[:, :1], w[:1].expand(far + 3, 16), ws[:, :1].expand(1, far + 3))):
        with pytest.raises(ValueError):
            call()


def test_a_stream_of_another_device_is_refused():
    import torch
    here = torch.cuda.current_device()
    other = types.SimpleNamespace(device=torch.device("cuda", here + 1), cuda_stream=0)
    x = torch.randn((5, 8), device="cuda")
    w, ws = map(_dev, _coded(3, 8))
    q, s = dss.quantize_mx4(x)
    y, v = torch.empty((5, 3), device="cuda"), torch.empty((5, 8), device="cuda")
    z, ids = torch.randn((5, 8), device="cuda"), torch.zeros((5, 2), dtype=torch.int64, device="cuda")
    losses, grad = torch.empty(5, device="cuda"), torch.empty_like(z)
    for call in (lambda **kw: dss.quantize_mx4(x, codes=q, scales=s, **kw), lambda **kw: dss.linear_mx4(x, w, ws, out=y, **kw),
                 lambda **kw: dss.matmul_mx4(q, s, w, ws, out=y, **kw), lambda **kw: dss.dequantize_mx4(q, s, 8, out=v, **kw),
                 lambda **kw: dss.distill(z, z[:, :2], ids, losses=losses, grad=grad, **kw)):
        with pytest.raises(ValueError):
            call(stream=other)
        for stream in (torch.cuda.Stream(), torch.cuda.current_stream(), torch.cuda.default_stream()):
            stream.wait_stream(torch.cuda.current_stream())
            call(stream=stream)
            torch.cuda.current_stream().wait_stream(stream)


def test_a_call_on_a_stream_that_is_not_the_current_one_owns_its_memory():
    """Outputs and workspaces made for a side stream are not handed to other work while it runs."""
    import torch
    side = torch.cuda.Stream()
    x = _x(4096, 700)
    w, ws = map(_dev, _coded(300, 700, 17))
    want = dss.linear_mx4(x, w, ws)
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(20):
        got.append(dss.linear_mx4(x, w, ws, stream=side))
        torch.empty(4096 * 400, dtype=torch.uint8, device="cuda").fill_(255)   # (as large as the workspace)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(want, y) for y in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 40), (2, 33), (40, 32), (65, 31), (255, 100), (256, 64), (257, 129), (700, 70), (1025, 32)])
def test_maps_whose_lines_start_anywhere(M, K, dtype):
    """Values to maps of every place within a line, for their first element and from channel to channel, and nothing beside
    them."""
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    codes, scales = _coded(M, K, 21)
    want = _dev(mx4.values(codes, scales, K).astype(np.float32)).to(dt).t()
    q, s = _dev(codes), _dev(scales)
    line = 128 // dt.itemsize
    for pad in (0, 1, line // 2, line - 1, line - M % line):
        for first in sorted({0, 1, line // 2 + 1, line - 1, line}):
            buf = torch.full((first + K * (M + pad) + line,), -77.0, dtype=dt, device="cuda")
            out = buf.as_strided((K, M), (M + pad, 1), first)
            dss.dequantize_mx4(q, s, K, out=out, planar=True)
            assert torch.equal(out, want), (pad, first)
            out.fill_(-77)
            assert bool((buf == -77).all()), (pad, first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 7, 31, 32, 33, 64, 96, 100, 127, 128, 129, 160])
def test_rows_of_few_blocks(K, dtype):
    """Around the count of blocks up to which a wave has several tokens: codes and values, and nothing beside them."""
    import torch
    for M in (1, 3, 127, 128, 129, 300):
        x = _x(M, K, "rows", dtype, seed=K)
        B = -(-K // 32)
        cbuf = torch.full((M + 2, 16 * B + 32), 55, dtype=torch.uint8, device="cuda")
        sbuf = torch.full((B + 2, M + 3), 55, dtype=torch.uint8, device="cuda")
        q, s = cbuf[1:M + 1, 16:16 + 16 * B], sbuf[1:B + 1, 1:M + 1]
        dss.quantize_mx4(x, q, s)
        want, wsc = mx4.quantize(_np(x))
        assert np.array_equal(q.cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), wsc)
        for pad in (0, 3, 128 // x.dtype.itemsize - K % 64):
            buf = torch.full((M + 2, K + max(pad, 0) + 1), -77.0, dtype=x.dtype, device="cuda")
            out = buf[1:M + 1, :K]
            dss.dequantize_mx4(q, s, K, out=out)
            assert np.array_equal(_np(out), mx4.values(want, wsc, K)), (M, pad)
            out.fill_(-77)
            assert bool((buf == -77).all())
        q.fill_(55), s.fill_(55)
        assert bool((cbuf == 55).all()) and bool((sbuf == 55).all())
