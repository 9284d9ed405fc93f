"""8-bit tokens and clipped gradients at the ends of their ranges: the most channels, the smallest factors, and
the parts of the products that ordinary sizes do not reach."""
import numpy as np
import pytest

from oracle import tokens
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
