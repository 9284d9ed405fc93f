"""Refusals of the gradient norm and clipping and of the 8-bit token calls, on the host: every
bad argument is named before anything is enqueued, so these need no GPU (the pointers are
never followed)."""
import ctypes

import numpy as np
import pytest

from paper_1508_06904_amd import dss

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 2, 3
PTR = 1 << 20                      # some 256-byte aligned address
VP = ctypes.c_void_p


def _list(*items):
    a = np.zeros(max(1, len(items)), dtype=[("data", "<u8"), ("count", "<i8"), ("dtype", "<i4"), ("reserved", "<i4")])
    for n, (data, count, dtype) in enumerate(items):
        a[n] = (data, count, dtype, 0)
    return a


def _clip(a, n, out=(PTR,), max_norm=1.0, norm=PTR, ws=PTR, wb=8192):
    outs = (VP * max(1, len(out)))(*out)
    return dss.lib().dss_clip_grads(VP(a.ctypes.data) if a is not None else None, outs, n, max_norm, VP(norm), VP(ws),
                                    wb, None)


GOOD = (PTR, 10, dss.DSS_F32)


@pytest.mark.parametrize("what,status,call", [
    ("negative n", INVALID, lambda: _clip(_list(GOOD), -1)),
    ("NULL list", INVALID, lambda: _clip(None, 1)),
    ("NULL norm", INVALID, lambda: _clip(_list(GOOD), 1, norm=None)),
    ("NULL data", INVALID, lambda: _clip(_list((0, 10, 0)), 1)),
    ("misaligned binary32", INVALID, lambda: _clip(_list((PTR + 2, 10, 0)), 1)),
    ("misaligned bfloat16", INVALID, lambda: _clip(_list((PTR + 1, 10, 1)), 1)),
    ("unknown dtype", UNSUPPORTED, lambda: _clip(_list((PTR, 10, 2)), 1)),
    ("negative count", INVALID, lambda: _clip(_list((PTR, -1, 0)), 1)),
    ("huge count", INVALID, lambda: _clip(_list((PTR, (1 << 40) + 1, 0)), 1)),
    ("NULL output", INVALID, lambda: _clip(_list(GOOD), 1, out=(None,))),
    ("misaligned output", INVALID, lambda: _clip(_list(GOOD), 1, out=(PTR + 1,))),
    ("negative max_norm", INVALID, lambda: _clip(_list(GOOD), 1, max_norm=-0.5)),
    ("NaN max_norm", INVALID, lambda: _clip(_list(GOOD), 1, max_norm=float("nan"))),
    ("NULL workspace", INVALID, lambda: _clip(_list(GOOD), 1, ws=None)),
    ("misaligned workspace", INVALID, lambda: _clip(_list(GOOD), 1, ws=PTR + 128)),
    ("small workspace", SHAPE, lambda: _clip(_list(GOOD), 1, wb=8191)),
])
def test_clip_refusals(what, status, call):
    assert call() == status, what
    assert dss.lib().dss_last_error()


def _quantize(x=PTR, dtype=0, M=4, K=8, ts=8, ks=1, codes=PTR, cs=8, scales=PTR):
    return dss.lib().dss_quantize_tokens(VP(x), dtype, M, K, ts, ks, VP(codes), cs, VP(scales), None)


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(x=None)), (INVALID, dict(x=PTR + 2)), (INVALID, dict(x=PTR + 1, dtype=1)),
    (INVALID, dict(codes=None)), (INVALID, dict(scales=None)), (INVALID, dict(scales=PTR + 2)),
    (INVALID, dict(M=-1)), (INVALID, dict(M=(1 << 40) + 1)), (INVALID, dict(K=0)), (INVALID, dict(K=-3)),
    (INVALID, dict(ts=-8)), (INVALID, dict(ts=1, ks=-4)), (INVALID, dict(cs=7)),
    (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(ts=16, ks=2)),
    (OK, dict(M=0, x=None, codes=None, scales=None)),
], ids=str)
def test_quantize_refusals(status, kw):
    assert _quantize(**kw) == status


def _matmul(codes=PTR, cs=64, scales=PTR, M=4, w=PTR, ws=64, wsc=PTR, N=8, K=64, bias=PTR, act=0, out=PTR, odt=0,
            ots=8, ocs=1, room=PTR, bytes=1 << 40):
    return dss.lib().dss_matmul_tokens(VP(codes), cs, VP(scales), M, VP(w), ws, VP(wsc), N, K, VP(bias), act, VP(out),
                                       odt, ots, ocs, VP(room), bytes, None)


def _linear(x=PTR, dt=0, M=4, ts=64, ks=1, w=PTR, ws=64, wsc=PTR, N=8, K=64, bias=PTR, act=0, out=PTR, odt=0, ots=8,
            ocs=1, room=PTR, bytes=1 << 40):
    return dss.lib().dss_linear_tokens(VP(x), dt, M, ts, ks, VP(w), ws, VP(wsc), N, K, VP(bias), act, VP(out), odt,
                                       ots, ocs, VP(room), bytes, None)


WIDE = dict(M=500, K=2500, ts=2500, ws=2500)       # sizes whose codes need a workspace

SHARED = [
    (INVALID, dict(w=None)), (INVALID, dict(wsc=None)), (INVALID, dict(wsc=PTR + 1)), (INVALID, dict(bias=PTR + 2)),
    (INVALID, dict(out=None)), (INVALID, dict(out=PTR + 2)), (INVALID, dict(out=PTR + 1, odt=1)),
    (INVALID, dict(M=-1)), (INVALID, dict(N=0)), (INVALID, dict(N=(1 << 20) + 1, ots=1 << 30)), (INVALID, dict(K=0)),
    (INVALID, dict(ws=63)), (INVALID, dict(act=3)), (INVALID, dict(act=-1)), (UNSUPPORTED, dict(odt=2)),
    (INVALID, dict(ots=7)), (INVALID, dict(ots=1, ocs=3)), (UNSUPPORTED, dict(ots=16, ocs=2)),
    (OK, dict(M=0)),
]


@pytest.mark.parametrize("status,kw", SHARED + [
    (INVALID, dict(codes=None)), (INVALID, dict(scales=None)), (INVALID, dict(scales=PTR + 2)), (INVALID, dict(cs=63)),
    (UNSUPPORTED, dict(K=131072, cs=131072, ws=131072)),
], ids=str)
def test_matmul_refusals(status, kw):
    assert _matmul(**kw) == status


@pytest.mark.parametrize("status,kw", SHARED + [
    (INVALID, dict(x=None)), (INVALID, dict(x=PTR + 2)), (UNSUPPORTED, dict(dt=3)), (INVALID, dict(ts=-64)),
    (UNSUPPORTED, dict(ts=128, ks=2)), (UNSUPPORTED, dict(K=131072, ts=131072, ws=131072)),
    (INVALID, dict(WIDE, room=None)), (INVALID, dict(WIDE, room=PTR + 16)), (SHAPE, dict(WIDE, bytes=100)),
], ids=str)
def test_linear_refusals(status, kw):
    assert _linear(**kw) == status


def test_workspace_query():
    need = ctypes.c_int64()
    q = dss.lib().dss_tokens_workspace
    assert q(500, 8, 2500, 0, ctypes.byref(need)) == OK and need.value >= 500 * 2500 + 500 * 4
    assert q(1 << 33, 8, 2500, 0, ctypes.byref(need)) == OK and need.value >= (1 << 33) * 2504
    assert q(0, 8, 64, 0, ctypes.byref(need)) == OK
    for bad in ((-1, 8, 64), (4, 0, 64), (4, 8, 0)):
        assert q(*bad, 0, ctypes.byref(need)) == INVALID
    assert q(4, 8, 64, 0, None) == INVALID


def test_binding_refuses_what_is_no_cuda_tensor():
    import torch
    x = torch.zeros(4, 8)
    for call in (lambda: dss.grad_norm([x]), lambda: dss.grad_norm(x), lambda: dss.clip_grads([1.0], 1.0),
                 lambda: dss.quantize_tokens(x), lambda: dss.quantize_tokens(x[0]),
                 lambda: dss.matmul_i8(x, x[:, 0], x, x[0]), lambda: dss.linear_i8(x, x, x[0])):
        with pytest.raises(ValueError):
            call()
