"""Layers in 4 bits in the calls that the sizes and layouts of test_gpu_mx4.py leave out.  Bounds as there."""
import numpy as np
import pytest

from oracle import mx4
from paper_1508_06904_amd import dss
from tests.test_gpu_mx4 import U, _check_layer, _coded, _dev, _np
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


# ---------------------------------------------------------------------------- codes that lie across

@pytest.mark.parametrize("planar", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (2, 5, 32), (9, 33, 100), (130, 70, 257), (600, 260, 128), (3000, 5, 96)])
def test_products_of_codes_that_lie_across(M, N, K, planar):
    """The bits of the same codes in rows, and the oracle's values: tokens adjacent, every second byte, a row repeated."""
    import torch
    tokens, weight = _coded(M, K, 3), _coded(N, K, 4)
    codes, scales, w, ws = map(_dev, tokens + weight)
    y = dss.matmul_mx4(codes, scales, w, ws, act="relu", planar=planar)
    _check_layer(y.t() if planar else y, mx4.values(*tokens), mx4.values(*weight), None, "relu")
    across = codes.t().contiguous().t()
    wide = torch.full((M, 2 * codes.shape[1] + 1), 0x77, dtype=torch.uint8, device="cuda")
    wide[:, 1::2] = codes
    side = torch.cuda.Stream()
    for c in (across, wide[:, 1::2], codes.t().contiguous().as_strided(codes.shape, (1, M))):
        assert torch.equal(c, codes)
        assert torch.equal(y, dss.matmul_mx4(c, scales, w, ws, act="relu", planar=planar))
        side.wait_stream(torch.cuda.current_stream())
        got = dss.matmul_mx4(c, scales, w, ws, act="relu", planar=planar, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(y, got)
    same = dss.matmul_mx4(codes[:1].expand(M, codes.shape[1]).t().contiguous().t(), scales[:, :1].expand(-1, M).contiguous(),
                          w, ws, act="relu", planar=planar)
    first = same[:, :1] if planar else same[:1]
    assert torch.equal(same, first.expand_as(same))


def test_products_of_codes_that_lie_across_in_a_graph():
    import torch
    tokens, weight = _coded(70, 130), _coded(33, 130, 1)
    codes, scales, w, ws = map(_dev, tokens + weight)
    across, y = codes.t().contiguous().t(), torch.empty((70, 33), device="cuda")
    dss.matmul_mx4(across, scales, w, ws, out=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dss.matmul_mx4(across, scales, w, ws, out=y)
    for n in range(3):
        codes.copy_(_dev(_coded(70, 130, n + 5)[0]))
        across.copy_(codes)
        y.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, dss.matmul_mx4(codes, scales, w, ws))


def test_other_codes_are_refused_as_before():
    import torch
    codes, scales, w, ws = map(_dev, _coded(6, 40) + _coded(5, 40, 1))
    odd = torch.empty((6, 40), dtype=torch.uint8, device="cuda")[:, :32]
    off = torch.empty((6, 48), dtype=torch.uint8, device="cuda")[:, 8:40]
    for c, s in ((odd, scales), (off, scales), (codes.t().contiguous().t()[:5], scales), (codes.t().contiguous().t()[:, :16], scales),
                 (codes[:1].expand(6, 32), scales), (codes.int(), scales), (codes.cpu().t().contiguous().t(), scales)):
        with pytest.raises(ValueError):
            dss.matmul_mx4(c, s, w, ws)
    with pytest.raises(ValueError):
        dss.matmul_mx4(codes, scales, w.t().contiguous().t(), ws)


# ---------------------------------------------------------------------------- one channel

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 2, 3, 7, 15, 16, 17, 40, 300])
def test_layers_of_one_channel_at_any_strides(M, dtype):
    """With one channel any two strides are allowed: every second window of a map, one token for all, tokens far apart."""
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    buf = torch.from_numpy(np.random.default_rng(M).standard_normal(9 * M + 20).astype(np.float32)).to("cuda").to(dt)
    weight = _coded(33, 1, 4)
    w, ws = map(_dev, weight)
    w8, ws8 = dss.quantize_tokens(_dev(mx4.values(*weight, 1).astype(np.float32)))
    every_second = buf[:2 * M][None][:, ::2].t()
    assert M == 1 or every_second.stride()[0] == 2
    for x in (every_second, buf.as_strided((M, 1), (0, 7)), buf.as_strided((M, 1), (9, 3)), buf.as_strided((M, 1), (3, 0)),
              buf.as_strided((M, 1), (5, 1)), buf.as_strided((M, 1), (1, 4))):
        for planar in (False, True):
            y = dss.linear_mx4(x, w, ws, planar=planar)
            _check_layer(y.t() if planar else y, mx4.values(*mx4.quantize(_np(x)), 1), mx4.values(*weight, 1))
            two = dss.matmul_mx4(*dss.quantize_mx4(x), w, ws, planar=planar)
            assert torch.equal(y, two)
            y = dss.linear_i8(x, w8, ws8, planar=planar)
            assert torch.equal(y, dss.linear_i8(x.contiguous(), w8, ws8, planar=planar))


# ---------------------------------------------------------------------------- both ends of binary32

def _at(M, N, K, target, seed=0):
    """Tokens and weights of random codes whose scales run over their range, block by block against each other, so that the
    largest sum of the products' magnitudes lies in 2^(target - 1) .. 2^target."""
    rng = np.random.default_rng([seed, M, N, K, abs(target)])
    (codes, _), (wcodes, _) = _coded(M, K, 20 + seed), _coded(N, K, 21 + seed)
    codes[:, ::16] |= 7                                 # (a 6 in each block: values are coded as they are held)
    B = -(-K // 32)
    j, i = rng.integers(0, 3, (B, M)), rng.integers(0, 3, (B, N))
    bytes_ = lambda e: (e + 127).astype(np.uint8)       # noqa: E731
    size = mx4.layer(mx4.values(codes, bytes_(-j)), mx4.values(wcodes, bytes_(-i)))[1].max()
    s = target - int(np.ceil(np.log2(size)))
    a = rng.integers(max(2, s), min(252, 250 + s) + 1, (B, 1))    # the tokens' bytes less j, the weights' 254 + s - a less i
    scales, wscales = (a - j).astype(np.uint8), (254 + s - a - i).astype(np.uint8)
    assert (254 + s - a - i).min() >= 0 and (254 + s - a - i).max() <= 254 and (a - j).min() >= 0
    return (codes, scales), (wcodes, wscales)


def _check_at(got, x, w):
    """As _check_layer; below 2^-126 a unit in the last place of an addition is 2^-149."""
    want, size = mx4.layer(x, w)
    n = -(-x.shape[1] // 128) + 8
    bound = 1.01 * U * (2 * n * size + np.abs(want)) + n * 2.0 ** -149
    off = np.abs(_np(got).astype(np.float64) - want)
    assert (off <= bound).all(), (np.argwhere(~(off <= bound))[:5], off.max())
    return want


FEW = [(1, 20, 130), (16, 64, 96), (300, 5, 100), (9, 700, 3000)]
TILES = [(70, 200, 96), (300, 300, 300), SHAPES[0][1]] + SHAPES[1] + SHAPES[2][:2]


@pytest.mark.parametrize("target", [127, 124, -120, -126, -128, -135])
@pytest.mark.parametrize("M,N,K", FEW + TILES)
def test_products_at_both_ends_of_binary32(M, N, K, target):
    import torch
    tokens, weight = _at(M, N, K, target)
    x, w = mx4.values(*tokens), mx4.values(*weight)
    y = dss.matmul_mx4(*map(_dev, tokens + weight))
    want = _check_at(y, x, w)
    assert 2.0 ** (target - 9) < np.abs(want).max() < 2.0 ** target
    planar = dss.matmul_mx4(*map(_dev, tokens + weight), planar=True)
    _check_at(planar.t(), x, w)
    # the same codes out of the values
    for v in (_dev(x.astype(np.float32)), _dev(x.T.astype(np.float32)).t()):
        codes, scales = dss.quantize_mx4(v[:, :K])
        assert np.array_equal(scales.cpu().numpy(), tokens[1])
        _check_at(dss.linear_mx4(v[:, :K], *map(_dev, weight)), x, w)


@pytest.mark.parametrize("target", [127, -126, -135])
@pytest.mark.parametrize("M,N,K", [(256, 5, 96), (900, 6, 128), (33000, 20, 300), (32900, 70, 512)])
def test_layers_of_maps_at_both_ends_of_binary32(M, N, K, target):
    import torch
    tokens, weight = _at(M, N, K, target, 1)
    x, w = mx4.values(*tokens), mx4.values(*weight)
    v = _dev(x[:, :K].T.astype(np.float32)).t()
    for planar in (False, True):
        y = dss.linear_mx4(v, *map(_dev, weight), planar=planar)
        _check_at(y.t() if planar else y, x, w)
    half = v.to(torch.bfloat16)                         # (exact: the codes have two bits, scales none; but below 2^-126
    assert torch.equal(half.float(), v)                 #  bfloat16 has 2^-133 for its last place)
    _check_at(dss.linear_mx4(half, *map(_dev, weight)), x, w)


@pytest.mark.parametrize("act", ["none", "relu", "tanh"])
@pytest.mark.parametrize("M,N,K", FEW + TILES + [(900, 6, 128)])
def test_sums_beyond_binary32_are_infinite(M, N, K, act):
    """Every second token's products are 36 2^118 of one sign, whose sum over a block is over 2^128; every third output's
    weights are negative. Other tokens stay finite."""
    import torch
    assert K >= 32
    codes, scales = _coded(M, K, 22)
    codes[::2] = mx4.quantize(np.full((1, K), 6.0))[0]
    scales[:, ::2] = 250
    wcodes, wscales = mx4.quantize(np.where(np.arange(N) % 3 == 2, -6.0, 6.0)[:, None] * np.ones((1, K)))
    wscales[:] = 254 + 118 - 250
    x, w = mx4.values(codes, scales), mx4.values(wcodes, wscales)
    want = np.where(np.arange(N) % 3 == 2, -np.inf, np.inf)
    want = np.maximum(want, 0.0) if act == "relu" else np.tanh(want) if act == "tanh" else want
    args = [_dev(a) for a in (codes, scales, wcodes, wscales)]
    v = torch.from_numpy(x[:, :K].astype(np.float32)).to("cuda")
    for y in (dss.matmul_mx4(*args, act=act), dss.matmul_mx4(*args, act=act, planar=True).t(),
              dss.matmul_mx4(*args, act=act, out_dtype=torch.bfloat16), dss.linear_mx4(v, *args[2:], act=act),
              dss.linear_mx4(v.t().contiguous().t(), *args[2:], act=act)):
        assert (_np(y[::2]) == want[None]).all()
        if act == "none" and y.dtype == torch.float32 and M > 1:
            _check_at(y[1::2], x[1::2], w)
