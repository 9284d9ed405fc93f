"""Refusals of the distillation call, on the host: every bad argument is named before anything is enqueued, so these need
no GPU (the pointers are never followed)."""
import ctypes

import pytest

from paper_1508_06904_amd import dss

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 2, 3
PTR = 1 << 20                      # some 256-byte aligned address
VP = ctypes.c_void_p


def _distill(z=PTR, dt=0, M=4, C=10, ts=10, cs=1, top=True, weights=PTR, T=1.0, scale=1.0, losses=PTR, grad=PTR, gts=10, gcs=1,
             room=PTR, bytes=1 << 22, **lists):
    fields = dict(logits=PTR, ids=PTR, token_stride=3, place_stride=1, id_token_stride=3, id_place_stride=1, count=3, dtype=0,
                  id_bytes=4, reserved=0)
    fields.update(lists)
    t = dss.TopLogits(**fields)
    return dss.lib().dss_distill_tokens(VP(z), dt, M, C, ts, cs, ctypes.byref(t) if top else None, VP(weights), T, scale,
                                        VP(losses), VP(grad), gts, gcs, VP(room), bytes, None)


LONG = dict(C=32769, ts=32769, gts=32769)              # sizes that need a workspace
WIDE = dict(C=129, ts=1, cs=4, gts=1, gcs=4)


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(z=None)), (INVALID, dict(z=PTR + 2)), (INVALID, dict(M=-1)), (INVALID, dict(C=0)), (INVALID, dict(ts=-1)),
    (UNSUPPORTED, dict(dt=2)), (UNSUPPORTED, dict(ts=20, cs=2)), (INVALID, dict(top=False)),
    (INVALID, dict(count=0)), (INVALID, dict(count=1025)), (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(id_bytes=2)),
    (INVALID, dict(token_stride=-1)), (INVALID, dict(place_stride=-1)), (INVALID, dict(id_token_stride=-1)),
    (INVALID, dict(id_place_stride=-1)), (INVALID, dict(logits=None)), (INVALID, dict(ids=None)), (INVALID, dict(logits=PTR + 2)),
    (INVALID, dict(logits=PTR + 1, dtype=1)), (INVALID, dict(ids=PTR + 4, id_bytes=8)),
    (INVALID, dict(T=0.0)), (INVALID, dict(T=-1.0)), (INVALID, dict(T=float("nan"))), (INVALID, dict(T=float("inf"))),
    (UNSUPPORTED, dict(T=2.0 ** -61)), (UNSUPPORTED, dict(T=2.0 ** 61)), (INVALID, dict(scale=float("inf"))),
    (INVALID, dict(scale=float("nan"))), (INVALID, dict(losses=None)), (INVALID, dict(losses=PTR + 2)),
    (INVALID, dict(weights=PTR + 1)), (INVALID, dict(grad=PTR + 2)), (INVALID, dict(gts=9)), (INVALID, dict(gts=1, gcs=4)),
    (INVALID, dict(gts=20, gcs=2)), (INVALID, dict(ts=1, cs=4, gts=10, gcs=1)), (INVALID, dict(ts=1, cs=4, gts=1, gcs=3)),
    (INVALID, dict(LONG, room=None)), (INVALID, dict(LONG, room=PTR + 8)), (SHAPE, dict(LONG, bytes=100)),
    (INVALID, dict(WIDE, room=None)), (SHAPE, dict(WIDE, bytes=100)), (INVALID, dict(grad=PTR, z=PTR, ts=20, gts=10)),
    (OK, dict(M=0, z=None, losses=None, grad=None, room=None)), (OK, dict(M=0, ts=1, cs=4, gts=1, gcs=4)),
], ids=str)
def test_refusals(status, kw):
    assert _distill(**kw) == status
    assert status == OK or dss.lib().dss_last_error()


def test_workspace_query():
    need = ctypes.c_int64()
    q = dss.lib().dss_distill_workspace
    for C, planar, none in ((1, 0, True), (32768, 0, True), (32769, 0, False), (128, 1, True), (129, 1, False),
                            (2 ** 31 - 1, 0, False), (2 ** 31 - 1, 1, False)):
        assert q(C, planar, ctypes.byref(need)) == OK and (need.value == 0) == none and 0 <= need.value <= 1 << 22
        assert dss.distill_workspace(C, bool(planar)) == need.value
    assert q(0, 0, ctypes.byref(need)) == INVALID and q(4, 0, None) == INVALID


def test_binding_refuses_what_is_no_cuda_tensor():
    import torch
    z = torch.zeros(4, 8)
    for bad in (z, z[0], [1.0]):
        with pytest.raises(ValueError):
            dss.distill(bad, z, torch.zeros(4, 8, dtype=torch.int64))
