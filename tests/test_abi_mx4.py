"""Refusals of the 4-bit token calls, on the host: every bad argument is named before anything is enqueued, so
these need no GPU (the pointers are never followed)."""
import ctypes

import pytest

from paper_1508_06904_amd import dss

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 2, 3
PTR = 1 << 20                      # some 256-byte aligned address
VP = ctypes.c_void_p


def _quantize(x=PTR, dtype=0, M=4, K=40, ts=40, ks=1, codes=PTR, cs=32, scales=PTR, ss=4):
    return dss.lib().dss_quantize_blocks(VP(x), dtype, M, K, ts, ks, VP(codes), cs, VP(scales), ss, None)


ROWS = [
    (INVALID, dict(codes=None)), (INVALID, dict(scales=None)), (INVALID, dict(codes=PTR + 8)), (INVALID, dict(cs=16)),
    (INVALID, dict(cs=40)), (INVALID, dict(ss=3)), (INVALID, dict(M=-1)), (INVALID, dict(M=(1 << 40) + 1, ss=1 << 41)),
]


@pytest.mark.parametrize("status,kw", ROWS + [
    (INVALID, dict(x=None)), (INVALID, dict(x=PTR + 2)), (INVALID, dict(x=PTR + 1, dtype=1)), (INVALID, dict(K=0)),
    (INVALID, dict(ts=-8)), (INVALID, dict(ts=1, ks=-4)), (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(ts=80, ks=2)),
    (OK, dict(M=0, x=None, codes=None, scales=None)),
], ids=str)
def test_quantize_refusals(status, kw):
    assert _quantize(**kw) == status
    assert status == OK or dss.lib().dss_last_error()


def _dequantize(codes=PTR, cs=32, scales=PTR, ss=4, M=4, K=40, out=PTR, dtype=0, ots=40, ocs=1):
    return dss.lib().dss_dequantize_blocks(VP(codes), cs, VP(scales), ss, M, K, VP(out), dtype, ots, ocs, None)


@pytest.mark.parametrize("status,kw", ROWS + [
    (INVALID, dict(out=None)), (INVALID, dict(out=PTR + 2)), (INVALID, dict(K=0)), (INVALID, dict(ots=39)),
    (INVALID, dict(ots=1, ocs=3)), (UNSUPPORTED, dict(ots=80, ocs=2)), (UNSUPPORTED, dict(dtype=2)),
    (OK, dict(M=0, out=None, codes=None, scales=None)),
], ids=str)
def test_dequantize_refusals(status, kw):
    assert _dequantize(**kw) == status


def _matmul(codes=PTR, cs=32, scales=PTR, ss=4, M=4, w=PTR, ws=32, wsc=PTR, wss=8, N=8, B=2, bias=PTR, act=0, out=PTR, odt=0,
            ots=8, ocs=1):
    return dss.lib().dss_matmul_blocks(VP(codes), cs, VP(scales), ss, M, VP(w), ws, VP(wsc), wss, N, B, VP(bias), act,
                                       VP(out), odt, ots, ocs, None)


def _linear(x=PTR, dt=0, M=4, ts=40, ks=1, w=PTR, ws=32, wsc=PTR, wss=8, N=8, K=40, bias=PTR, act=0, out=PTR, odt=0, ots=8,
            ocs=1, room=PTR, bytes=1 << 40):
    return dss.lib().dss_linear_blocks(VP(x), dt, M, ts, ks, VP(w), ws, VP(wsc), wss, N, K, VP(bias), act, VP(out), odt,
                                       ots, ocs, VP(room), bytes, None)


SHARED = [
    (INVALID, dict(w=None)), (INVALID, dict(wsc=None)), (INVALID, dict(w=PTR + 8)), (INVALID, dict(bias=PTR + 2)),
    (INVALID, dict(ws=16)), (INVALID, dict(ws=40)), (INVALID, dict(wss=7)),
    (INVALID, dict(out=None)), (INVALID, dict(out=PTR + 2)), (INVALID, dict(out=PTR + 1, odt=1)),
    (INVALID, dict(M=-1)), (INVALID, dict(N=0)), (INVALID, dict(N=(1 << 20) + 1, ots=1 << 30, wss=1 << 30)),
    (INVALID, dict(act=3)), (INVALID, dict(act=-1)), (UNSUPPORTED, dict(odt=2)),
    (INVALID, dict(ots=7)), (INVALID, dict(ots=1, ocs=3)), (UNSUPPORTED, dict(ots=16, ocs=2)),
    (OK, dict(M=0)),
]


@pytest.mark.parametrize("status,kw", SHARED + ROWS + [(INVALID, dict(B=0)), (INVALID, dict(B=-1))], ids=str)
def test_matmul_refusals(status, kw):
    assert _matmul(**kw) == status


WIDE = dict(M=500, K=2500, ts=2500, ws=1264)       # sizes whose codes need a workspace


@pytest.mark.parametrize("status,kw", SHARED + [
    (INVALID, dict(x=None)), (INVALID, dict(x=PTR + 2)), (UNSUPPORTED, dict(dt=3)), (INVALID, dict(ts=-64)),
    (INVALID, dict(K=0)), (UNSUPPORTED, dict(ts=128, ks=2)),
    (INVALID, dict(WIDE, room=None)), (INVALID, dict(WIDE, room=PTR + 16)), (SHAPE, dict(WIDE, bytes=100)),
], ids=str)
def test_linear_refusals(status, kw):
    assert _linear(**kw) == status


def test_workspace_query():
    need = ctypes.c_int64()
    q = dss.lib().dss_blocks_workspace
    assert q(500, 8, 2500, 0, ctypes.byref(need)) == OK and need.value >= 500 * 79 * 17
    assert q(500, 8, 2500, 2, ctypes.byref(need)) == OK and need.value == 0
    assert q(1 << 33, 8, 2500, 0, ctypes.byref(need)) == OK and need.value >= (1 << 33) * 79 * 17
    assert q(0, 8, 64, 0, ctypes.byref(need)) == OK
    for bad in ((-1, 8, 64), (4, 0, 64), (4, 8, 0), (1 << 40, 8, 2 ** 31 - 1)):
        assert q(*bad, 0, ctypes.byref(need)) == INVALID
    assert q(4, 8, 64, 3, ctypes.byref(need)) == INVALID
    assert q(4, 8, 64, 0, None) == INVALID


def test_binding_refuses_what_is_no_cuda_tensor():
    import torch
    x, c = torch.zeros(4, 32), torch.zeros(4, 16, dtype=torch.uint8)
    for call in (lambda: dss.quantize_mx4(x), lambda: dss.quantize_mx4(x[0]), lambda: dss.dequantize_mx4(c, c[:, 0]),
                 lambda: dss.matmul_mx4(c, c, c, c), lambda: dss.linear_mx4(x, c, c)):
        with pytest.raises(ValueError):
            call()
