"""Layers in 4 bits in the calls that the sizes and layouts of test_gpu_mx4.py leave out.  Bounds as there."""
import numpy as np
import pytest

from oracle import mx4
from paper_1508_06904_amd import dss
from tests.test_gpu_mx4 import _check_layer, _coded, _dev, _np

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
