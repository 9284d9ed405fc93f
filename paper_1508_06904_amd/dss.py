"""Python binding of libdss.so (include/dss.h): argument marshalling only.

Every step of the dense evaluation runs in the library's HIP kernels; torch is
used here for device memory (tensors whose data pointers are handed to the C
ABI) and for the current HIP stream.  There is no fallback: if libdss.so is
missing or a call fails, a `DssError` is raised.

Layers are the dicts produced by `workloads`:
  {"kind": "conv", "cin", "cout", "fh", "fw", "act", "weight": [cout][cin][fh][fw], "bias": [cout]}
  {"kind": "maxpool", "kh", "kw"}
"""
from __future__ import annotations

import array
import ctypes
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdss.so")

DSS_F32, DSS_BF16 = 0, 1
DTYPES = {"f32": DSS_F32, "bf16": DSS_BF16}
ACTS = {"none": 0, "relu": 1, "tanh": 2}


class DssError(RuntimeError):
    def __init__(self, status, what, detail):
        super().__init__("%s failed with status %d (%s): %s" % (what, status, _STATUS.get(status, "?"), detail))
        self.status = status


_STATUS = {0: "ok", 1: "invalid", 2: "shape", 3: "unsupported", 4: "nomem", 5: "hip"}


class Layer(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("cin", ctypes.c_int32), ("cout", ctypes.c_int32),
                ("fh", ctypes.c_int32), ("fw", ctypes.c_int32), ("act", ctypes.c_int32),
                ("kh", ctypes.c_int32), ("kw", ctypes.c_int32),
                ("weight", ctypes.POINTER(ctypes.c_float)), ("bias", ctypes.POINTER(ctypes.c_float))]


class Geometry(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("ndim", "in_c", "out_c", "n_chain", "B_h", "B_w", "K_h", "K_w", "r_h", "r_w",
                 "D_h", "D_w", "out_h", "out_w", "dtype", "ell", "step_h", "step_w", "trim_h", "trim_w")] + \
               [("workspace_bytes", ctypes.c_int64), ("conv_flops", ctypes.c_double),
                ("pool_bytes", ctypes.c_double), ("total_bytes", ctypes.c_double)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class LayerGeometry(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("c_h", "c_w", "k_h", "k_w", "kstar_h", "kstar_w", "u_h", "u_w", "U_h", "U_w", "F",
                 "channels", "has_conv", "has_pool", "relaxed", "reserved")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_ if n != "reserved"}


class LaunchRecord(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_char_p), ("chain_layer", ctypes.c_int32), ("tile_mode", ctypes.c_int32),
                ("ms", ctypes.c_double), ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


GRAD_NORM_WORKSPACE_BYTES = 8192

EXPORTS = ("dss_chain_geometry", "dss_chain_layer_geometry", "dss_plan_create", "dss_plan_destroy",
           "dss_plan_geometry", "dss_plan_layer_geometry", "dss_eval_dense", "dss_eval_mixed", "dss_eval_slide",
           "dss_chain_stride_geometry", "dss_plan_stride_geometry", "dss_eval_stride", "dss_chain_dilate_geometry",
           "dss_plan_dilate_geometry", "dss_eval_dilate", "dss_chain_backward_geometry",
           "dss_plan_backward_geometry", "dss_backward_dense", "dss_eval_dense_noalloc", "dss_frag", "dss_defrag",
           "dss_grad_norm", "dss_clip_grads", "dss_quantize_tokens", "dss_tokens_workspace", "dss_matmul_tokens",
           "dss_linear_tokens", "dss_plan_set_timing", "dss_plan_timings", "dss_status_string", "dss_last_error", "dss_version")

_lib = None


def _torch_device_first():
    """With torch in the process there are two HIP runtimes: torch's own copy and
    the system one that libdss.so links.  If the system one brings the device up
    first, torch's then reports no device; bringing torch's up first (when torch
    is installed and sees a device) works in either use.  Nothing happens on a
    machine without a GPU."""
    try:
        import torch
    except ImportError:
        return
    if torch.cuda.is_available():
        torch.cuda.init()


def lib():
    """Load libdss.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise DssError(-1, "loading libdss.so", "%s does not exist; run __graft_entry__.build()" % LIB_PATH)
        _torch_device_first()
        L = ctypes.CDLL(LIB_PATH)
        P, I32, I64, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        L.dss_chain_geometry.argtypes = [P(Layer), I32, I32, I32, I32, I32, I32, I32, P(Geometry)]
        L.dss_chain_layer_geometry.argtypes = [P(Layer), I32, I32, I32, I32, I32, I32, I32, P(LayerGeometry)]
        L.dss_plan_create.argtypes = [P(Layer), I32, I32, I32, I32, P(VP)]
        L.dss_plan_destroy.argtypes = [VP]
        L.dss_plan_destroy.restype = None
        L.dss_plan_geometry.argtypes = [VP, I32, I32, I32, P(Geometry)]
        L.dss_plan_layer_geometry.argtypes = [VP, I32, I32, I32, I32, P(LayerGeometry)]
        L.dss_eval_dense.argtypes = [VP, VP, I32, I32, VP, VP, I64, VP]
        L.dss_eval_mixed.argtypes = [VP, VP, I32, I32, I32, VP, VP, I64, VP]
        L.dss_eval_slide.argtypes = [VP, VP, I32, I32, I32, I32, VP, VP, I64, VP]
        L.dss_chain_stride_geometry.argtypes = [P(Layer), I32, I32, I32, I32, I32, P(I64), P(ctypes.c_double)]
        L.dss_plan_stride_geometry.argtypes = [VP, I32, P(I64), P(ctypes.c_double)]
        L.dss_eval_stride.argtypes = [VP, VP, I32, I32, I64, I32, VP, VP, I64, VP]
        L.dss_chain_dilate_geometry.argtypes = [P(Layer), I32, I32, I32, I32, I32, I32, I32, P(I32), P(I32), P(I64),
                                                P(ctypes.c_double)]
        L.dss_plan_dilate_geometry.argtypes = [VP, I32, I32, I32, P(I32), P(I32), P(I64), P(ctypes.c_double)]
        L.dss_eval_dilate.argtypes = [VP, VP, I32, I32, I32, VP, VP, I64, VP]
        L.dss_chain_backward_geometry.argtypes = [P(Layer), I32, I32, I32, I32, I32, I32, P(I64), P(I64), P(I64),
                                                  P(ctypes.c_double)]
        L.dss_plan_backward_geometry.argtypes = [VP, I32, I32, I32, P(I64), P(I64), P(I64), P(ctypes.c_double)]
        L.dss_backward_dense.argtypes = [VP, VP, I32, I32, VP, VP, VP, VP, VP, I64, VP]
        L.dss_eval_dense_noalloc.argtypes = [VP, VP, I32, I32, VP, VP]
        L.dss_frag.argtypes = [I32, I32, I32, I32, I32, I32, I32, I32, VP, VP, VP]
        L.dss_defrag.argtypes = [I32, I32, I32, I32, I32, I32, I32, I32, VP, VP, VP]
        L.dss_grad_norm.argtypes = [VP, I32, VP, VP, I64, VP]
        L.dss_clip_grads.argtypes = [VP, VP, I32, ctypes.c_float, VP, VP, I64, VP]
        L.dss_quantize_tokens.argtypes = [VP, I32, I64, I32, I64, I64, VP, I64, VP, VP]
        L.dss_tokens_workspace.argtypes = [I64, I32, I32, I32, P(I64)]
        L.dss_matmul_tokens.argtypes = [VP, I64, VP, I64, VP, I64, VP, I32, I32, VP, I32, VP, I32, I64, I64, VP, I64, VP]
        L.dss_linear_tokens.argtypes = [VP, I32, I64, I64, I64, VP, I64, VP, I32, I32, VP, I32, VP, I32, I64, I64, VP,
                                        I64, VP]
        L.dss_plan_set_timing.argtypes = [VP, I32]
        L.dss_plan_timings.argtypes = [VP, P(LaunchRecord), I32, P(I32)]
        L.dss_status_string.argtypes = [I32]
        L.dss_status_string.restype = ctypes.c_char_p
        L.dss_last_error.argtypes = []
        L.dss_last_error.restype = ctypes.c_char_p
        L.dss_version.argtypes = []
        L.dss_version.restype = ctypes.c_char_p
        for name in ("dss_chain_geometry", "dss_chain_layer_geometry", "dss_plan_create", "dss_plan_geometry",
                     "dss_plan_layer_geometry", "dss_eval_dense", "dss_eval_mixed", "dss_eval_slide", "dss_frag",
                     "dss_defrag", "dss_plan_set_timing", "dss_plan_timings", "dss_plan_stride_geometry",
                     "dss_chain_stride_geometry", "dss_eval_stride", "dss_chain_dilate_geometry",
                     "dss_plan_dilate_geometry", "dss_eval_dilate", "dss_chain_backward_geometry",
                     "dss_plan_backward_geometry", "dss_backward_dense", "dss_eval_dense_noalloc", "dss_grad_norm",
                     "dss_clip_grads", "dss_quantize_tokens", "dss_tokens_workspace", "dss_matmul_tokens",
                     "dss_linear_tokens"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status, what):
    if status != 0:
        raise DssError(status, what, lib().dss_last_error().decode())


class _LayerArray:
    """ctypes dss_layer array plus the binary32 weight copies it points into."""

    def __init__(self, layers):
        self.keep = []
        self.arr = (Layer * max(1, len(layers)))()
        for t, l in enumerate(layers):
            if l["kind"] == "conv":
                w = np.ascontiguousarray(l["weight"], dtype=np.float32)
                assert w.shape == (l["cout"], l["cin"], l["fh"], l["fw"])
                b = None if l.get("bias") is None else np.ascontiguousarray(l["bias"], dtype=np.float32)
                self.keep += [w, b]
                self.arr[t] = Layer(0, l["cin"], l["cout"], l["fh"], l["fw"], ACTS[l["act"]], 1, 1,
                                    w.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                    b.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) if b is not None
                                    else ctypes.POINTER(ctypes.c_float)())
            else:
                self.arr[t] = Layer(1, 0, 0, 1, 1, 0, l["kh"], l["kw"], ctypes.POINTER(ctypes.c_float)(),
                                    ctypes.POINTER(ctypes.c_float)())
        self.n = len(layers)


def chain_geometry(layers, ndim, in_channels, H, W, dtype="f32", ell=0):
    la = _LayerArray(layers)
    g = Geometry()
    _check(lib().dss_chain_geometry(la.arr, la.n, ndim, in_channels, DTYPES[dtype], H, W, ell, ctypes.byref(g)),
           "dss_chain_geometry")
    return g.as_dict()


def chain_layer_geometry(layers, ndim, in_channels, H, W, j, ell=0):
    la = _LayerArray(layers)
    g = LayerGeometry()
    _check(lib().dss_chain_layer_geometry(la.arr, la.n, ndim, in_channels, H, W, ell, j, ctypes.byref(g)),
           "dss_chain_layer_geometry")
    return g.as_dict()


def chain_stride_geometry(layers, ndim, in_channels, count, dtype="f32"):
    """(workspace bytes, conv flops) of the patch-by-patch baseline on `count` windows (host only)."""
    la = _LayerArray(layers)
    ws = ctypes.c_int64()
    fl = ctypes.c_double()
    _check(lib().dss_chain_stride_geometry(la.arr, la.n, ndim, in_channels, DTYPES[dtype], count, ctypes.byref(ws),
                                           ctypes.byref(fl)), "dss_chain_stride_geometry")
    return ws.value, fl.value


def chain_dilate_geometry(layers, ndim, in_channels, H, W, j, dtype="f32"):
    """(V_h, V_w, workspace bytes, conv flops) of the dilated evaluation after layer j (host only)."""
    la = _LayerArray(layers)
    vh, vw, ws, fl = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int64(), ctypes.c_double()
    _check(lib().dss_chain_dilate_geometry(la.arr, la.n, ndim, in_channels, DTYPES[dtype], H, W, j, ctypes.byref(vh),
                                           ctypes.byref(vw), ctypes.byref(ws), ctypes.byref(fl)),
           "dss_chain_dilate_geometry")
    return vh.value, vw.value, ws.value, fl.value


def chain_backward_geometry(layers, ndim, in_channels, H, W, with_signal_grad=True):
    """(workspace bytes, weight-gradient floats, bias-gradient floats, flops) of the backward pass (host only)."""
    la = _LayerArray(layers)
    ws, wf, bf, fl = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_double()
    _check(lib().dss_chain_backward_geometry(la.arr, la.n, ndim, in_channels, H, W, 1 if with_signal_grad else 0,
                                             ctypes.byref(ws), ctypes.byref(wf), ctypes.byref(bf), ctypes.byref(fl)),
           "dss_chain_backward_geometry")
    return ws.value, wf.value, bf.value, fl.value


def _stream(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr())


def _check_buffer(t, what, dtype, numel=None, min_numel=None, device=None):
    """Raises ValueError unless t is a contiguous CUDA tensor of `dtype` (a torch
    dtype, or an element size in bytes) with exactly `numel` (or at least
    `min_numel`) elements, on `device` if given.  The C ABI takes no sizes for
    these buffers, so a wrong one would mean out-of-bounds device accesses."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor" % what)
    if isinstance(dtype, int):
        if t.element_size() != dtype or t.is_complex():
            raise ValueError("%s must have %d-byte elements (got %s)" % (what, dtype, t.dtype))
    elif t.dtype != dtype:
        raise ValueError("%s must be %s (got %s)" % (what, dtype, t.dtype))
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, the signal on %s" % (what, t.device, device))
    if numel is not None and t.numel() != numel:
        raise ValueError("%s has %d elements, %d expected" % (what, t.numel(), numel))
    if min_numel is not None and t.numel() < min_numel:
        raise ValueError("%s has %d elements, at least %d needed" % (what, t.numel(), min_numel))


def _workspace_args(ws, device):
    """(pointer, bytes) of a caller workspace, or (NULL, 0): the plan's own."""
    if ws is None:
        return ctypes.c_void_p(None), 0
    import torch
    if not isinstance(ws, torch.Tensor) or not ws.is_cuda or not ws.is_contiguous() or ws.device != device:
        raise ValueError("workspace must be a contiguous CUDA tensor on the signal's device")
    return _ptr(ws), ws.numel() * ws.element_size()


class Plan:
    """A dss plan on the current device."""

    def __init__(self, layers, ndim, in_channels, dtype="f32"):
        self.layers = layers
        self.ndim = ndim
        self.in_channels = in_channels
        self.dtype = dtype
        la = _LayerArray(layers)
        h = ctypes.c_void_p()
        _check(lib().dss_plan_create(la.arr, la.n, ndim, in_channels, DTYPES[dtype], ctypes.byref(h)),
               "dss_plan_create")
        self.handle = h

    @classmethod
    def from_workload(cls, wl):
        return cls(wl.layers, wl.ndim, wl.x.shape[0], wl.dtype)

    def close(self):
        if getattr(self, "handle", None):
            lib().dss_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def geometry(self, H, W, ell=0):
        g = Geometry()
        _check(lib().dss_plan_geometry(self.handle, H, W, ell, ctypes.byref(g)), "dss_plan_geometry")
        return g.as_dict()

    def layer_geometry(self, H, W, j, ell=0):
        g = LayerGeometry()
        _check(lib().dss_plan_layer_geometry(self.handle, H, W, ell, j, ctypes.byref(g)), "dss_plan_layer_geometry")
        return g.as_dict()

    def workspace(self, H, W, device=None, ell=0):
        """A new device workspace (uint8 tensor) large enough for dss_eval_dense /
        dss_eval_mixed on an H x W signal at mixed level ell.  Calls that pass no
        workspace use the plan's own one inside the library instead."""
        import torch
        need = self.geometry(H, W, ell)["workspace_bytes"]
        return torch.empty(max(need, 256), dtype=torch.uint8, device=device or "cuda")

    def _check_signal(self, signal):
        import torch
        want = torch.float32 if self.dtype == "f32" else torch.bfloat16
        if not signal.is_cuda or signal.dtype != want or not signal.is_contiguous() or signal.dim() != 3:
            raise ValueError("signal must be a contiguous CUDA %s tensor [C][H][W]" % want)
        if signal.shape[0] != self.in_channels:
            raise ValueError("signal has %d channels, plan expects %d" % (signal.shape[0], self.in_channels))

    def eval_dense(self, signal, out=None, workspace=None, stream=None):
        import torch
        self._check_signal(signal)
        _, H, W = signal.shape
        g = self.geometry(H, W)
        if out is None:
            out = torch.empty((g["out_c"], g["out_h"], g["out_w"]), dtype=torch.float32, device=signal.device)
        _check_buffer(out, "out", torch.float32, g["out_c"] * g["out_h"] * g["out_w"], device=signal.device)
        wp, wb = _workspace_args(workspace, signal.device)
        _check(lib().dss_eval_dense(self.handle, _ptr(signal), H, W, _ptr(out), wp, wb, _stream(stream)),
               "dss_eval_dense")
        return out

    def eval_dense_noalloc(self, signal, out, stream=None):
        """dss_eval_dense_noalloc: the dense evaluation in the library's fixed
        scratch array (no device allocation, `out` must be given)."""
        import torch
        self._check_signal(signal)
        _, H, W = signal.shape
        g = self.geometry(H, W)
        _check_buffer(out, "out", torch.float32, g["out_c"] * g["out_h"] * g["out_w"], device=signal.device)
        _check(lib().dss_eval_dense_noalloc(self.handle, _ptr(signal), H, W, _ptr(out), _stream(stream)),
               "dss_eval_dense_noalloc")
        return out

    def eval_mixed(self, signal, ell, out=None, workspace=None, stream=None):
        import torch
        self._check_signal(signal)
        _, H, W = signal.shape
        g = self.geometry(H, W, ell)
        if out is None:
            out = torch.empty((g["out_c"], g["out_h"], g["out_w"]), dtype=torch.float32, device=signal.device)
        _check_buffer(out, "out", torch.float32, g["out_c"] * g["out_h"] * g["out_w"], device=signal.device)
        wp, wb = _workspace_args(workspace, signal.device)
        _check(lib().dss_eval_mixed(self.handle, _ptr(signal), H, W, ell, _ptr(out), wp, wb, _stream(stream)),
               "dss_eval_mixed")
        return out

    def eval_slide(self, signal, j, out=None, workspace=None, stream=None, ell=0):
        import torch
        self._check_signal(signal)
        _, H, W = signal.shape
        lg = self.layer_geometry(H, W, j, ell)
        if out is None:
            out = torch.empty((lg["F"], lg["channels"], lg["U_h"], lg["U_w"]), dtype=torch.float32,
                              device=signal.device)
        _check_buffer(out, "out", torch.float32, lg["F"] * lg["channels"] * lg["U_h"] * lg["U_w"],
                      device=signal.device)
        wp, wb = _workspace_args(workspace, signal.device)
        _check(lib().dss_eval_slide(self.handle, _ptr(signal), H, W, ell, j, _ptr(out), wp, wb, _stream(stream)),
               "dss_eval_slide")
        return out

    def dilate_geometry(self, H, W, j):
        """(V_h, V_w, workspace bytes, conv flops) of eval_dilate after layer j."""
        vh, vw, ws, fl = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int64(), ctypes.c_double()
        _check(lib().dss_plan_dilate_geometry(self.handle, H, W, j, ctypes.byref(vh), ctypes.byref(vw),
                                              ctypes.byref(ws), ctypes.byref(fl)), "dss_plan_dilate_geometry")
        return vh.value, vw.value, ws.value, fl.value

    def eval_dilate(self, signal, j=None, out=None, workspace=None, stream=None):
        """EvalDilate_j (default j = L, the dense output) as planar binary32 [C_j][V_h][V_w]."""
        import torch
        self._check_signal(signal)
        _, H, W = signal.shape
        n_chain = self.geometry(H, W)["n_chain"]
        j = n_chain if j is None else j
        vh, vw, _, _ = self.dilate_geometry(H, W, j)
        C = self.in_channels if j == 0 else self.layer_geometry(H, W, j)["channels"]
        if out is None:
            out = torch.empty((C, vh, vw), dtype=torch.float32, device=signal.device)
        _check_buffer(out, "out", torch.float32, C * vh * vw, device=signal.device)
        wp, wb = _workspace_args(workspace, signal.device)
        _check(lib().dss_eval_dilate(self.handle, _ptr(signal), H, W, j, _ptr(out), wp, wb, _stream(stream)),
               "dss_eval_dilate")
        return out

    def backward_geometry(self, H, W, with_signal_grad=True):
        """(workspace bytes, weight-gradient floats, bias-gradient floats, flops) of backward()."""
        ws, wf, bf, fl = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_double()
        _check(lib().dss_plan_backward_geometry(self.handle, H, W, 1 if with_signal_grad else 0, ctypes.byref(ws),
                                                ctypes.byref(wf), ctypes.byref(bf), ctypes.byref(fl)),
               "dss_plan_backward_geometry")
        return ws.value, wf.value, bf.value, fl.value

    def backward(self, signal, grad_out, with_signal_grad=True, grad_weight=None, grad_bias=None, workspace=None,
                 stream=None):
        """Gradients of sum(grad_out * eval_dense(signal)).  Returns (flat weight
        gradients, flat bias gradients, signal gradient or None) as CUDA tensors;
        `split_grads` cuts the flat ones per convolution."""
        import torch
        self._check_signal(signal)
        _, H, W = signal.shape
        _, wf, bf, _ = self.backward_geometry(H, W, with_signal_grad)
        g = self.geometry(H, W)
        dev = signal.device
        if grad_weight is None:
            grad_weight = torch.empty(max(wf, 1), dtype=torch.float32, device=dev)
        if grad_bias is None:
            grad_bias = torch.empty(max(bf, 1), dtype=torch.float32, device=dev)
        gx = torch.empty_like(signal) if with_signal_grad else None
        _check_buffer(grad_out, "grad_out", torch.float32, g["out_c"] * g["out_h"] * g["out_w"], device=dev)
        _check_buffer(grad_weight, "grad_weight", torch.float32, min_numel=wf, device=dev)
        _check_buffer(grad_bias, "grad_bias", torch.float32, min_numel=bf, device=dev)
        wp, wb = _workspace_args(workspace, dev)
        _check(lib().dss_backward_dense(self.handle, _ptr(signal), H, W, _ptr(grad_out), _ptr(grad_weight),
                                        _ptr(grad_bias), _ptr(gx) if gx is not None else None, wp, wb,
                                        _stream(stream)), "dss_backward_dense")
        return grad_weight, grad_bias, gx

    def split_grads(self, grad_weight, grad_bias):
        """Per-convolution views [cout][cin][fh][fw] and [cout] of the flat gradients."""
        ws, bs, ow, ob = [], [], 0, 0
        for l in self.layers:
            if l["kind"] != "conv":
                continue
            n = l["cout"] * l["cin"] * l["fh"] * l["fw"]
            ws.append(grad_weight[ow:ow + n].view(l["cout"], l["cin"], l["fh"], l["fw"]))
            bs.append(grad_bias[ob:ob + l["cout"]])
            ow += n
            ob += l["cout"]
        return ws, bs

    def stride_geometry(self, count):
        """(workspace bytes, conv flops) of eval_stride on a batch of `count` windows."""
        ws = ctypes.c_int64()
        fl = ctypes.c_double()
        _check(lib().dss_plan_stride_geometry(self.handle, count, ctypes.byref(ws), ctypes.byref(fl)),
               "dss_plan_stride_geometry")
        return ws.value, fl.value

    def eval_stride(self, signal, first, count, out=None, workspace=None, stream=None):
        """Patch-by-patch baseline on windows first..first+count-1 (row-major);
        writes those positions of `out` ([out_c][H-B_h+1][W-B_w+1], allocated if None)."""
        import torch
        self._check_signal(signal)
        _, H, W = signal.shape
        g = self.geometry(H, W)
        if out is None:
            out = torch.zeros((g["out_c"], g["out_h"], g["out_w"]), dtype=torch.float32, device=signal.device)
        _check_buffer(out, "out", torch.float32, g["out_c"] * g["out_h"] * g["out_w"], device=signal.device)
        wp, wb = _workspace_args(workspace, signal.device)
        _check(lib().dss_eval_stride(self.handle, _ptr(signal), H, W, first, count, _ptr(out), wp, wb,
                                     _stream(stream)), "dss_eval_stride")
        return out

    def set_timing(self, on=True):
        _check(lib().dss_plan_set_timing(self.handle, 1 if on else 0), "dss_plan_set_timing")

    def timings(self):
        n = ctypes.c_int32()
        _check(lib().dss_plan_timings(self.handle, None, 0, ctypes.byref(n)), "dss_plan_timings")
        recs = (LaunchRecord * max(1, n.value))()
        _check(lib().dss_plan_timings(self.handle, recs, n.value, ctypes.byref(n)), "dss_plan_timings")
        return [{"kernel": r.kernel.decode(), "layer": r.chain_layer, "ms": r.ms, "flops": r.flops,
                 "bytes": r.bytes, "tile_mode": r.tile_mode} for r in recs[: n.value]]


def frag(x, k_h, k_w, S_h, S_w, out=None, stream=None):
    """dss_frag on a CUDA tensor [S_h*S_w][C][H][W] of 4- or 2-byte elements."""
    import torch
    if not isinstance(x, torch.Tensor) or x.dim() != 4 or x.element_size() not in (2, 4):
        raise ValueError("x must be a 4-D tensor [S_h*S_w][C][H][W] of 2- or 4-byte elements")
    S, C, H, W = x.shape
    if S != S_h * S_w:
        raise ValueError("x holds %d fragments, S_h * S_w = %d" % (S, S_h * S_w))
    _check_buffer(x, "x", x.element_size())
    dt = DSS_BF16 if x.element_size() == 2 else DSS_F32
    if out is None:
        out = torch.empty((k_h * S_h * k_w * S_w, C, H // k_h, W // k_w), dtype=x.dtype, device=x.device)
    # extents that k does not divide are the library's DSS_E_SHAPE, before any access
    if k_h > 0 and k_w > 0 and H % k_h == 0 and W % k_w == 0:
        _check_buffer(out, "out", x.element_size(), S * C * H * W, device=x.device)
    _check(lib().dss_frag(k_h, k_w, S_h, S_w, C, H, W, dt, _ptr(x), _ptr(out), _stream(stream)), "dss_frag")
    return out


def defrag(x, k_h, k_w, S_h, S_w, out=None, stream=None):
    """dss_defrag on a CUDA tensor [(k_h*S_h)*(k_w*S_w)][C][H][W]."""
    import torch
    if not isinstance(x, torch.Tensor) or x.dim() != 4 or x.element_size() not in (2, 4):
        raise ValueError("x must be a 4-D tensor [(k_h*S_h)*(k_w*S_w)][C][H][W] of 2- or 4-byte elements")
    F, C, H, W = x.shape
    if F != k_h * S_h * k_w * S_w:
        raise ValueError("x holds %d fragments, (k_h * S_h) * (k_w * S_w) = %d" % (F, k_h * S_h * k_w * S_w))
    _check_buffer(x, "x", x.element_size())
    dt = DSS_BF16 if x.element_size() == 2 else DSS_F32
    if out is None:
        out = torch.empty((S_h * S_w, C, H * k_h, W * k_w), dtype=x.dtype, device=x.device)
    _check_buffer(out, "out", x.element_size(), F * C * H * W, device=x.device)
    _check(lib().dss_defrag(k_h, k_w, S_h, S_w, C, H, W, dt, _ptr(x), _ptr(out), _stream(stream)), "dss_defrag")
    return out


# ---------------------------------------------------------------------------- gradient norm and clipping
#
# These calls and the token calls below run for a few microseconds on small inputs, about what
# their arguments' checks cost here: each check is made once, with torch's cheapest query for it.

_DTYPE_CODE = None      # torch dtype -> dss_dtype, once torch is there


def _dtype_codes():
    global _DTYPE_CODE
    if _DTYPE_CODE is None:
        import torch
        _DTYPE_CODE = {torch.float32: DSS_F32, torch.bfloat16: DSS_BF16}
    return _DTYPE_CODE


def _launch(stream):
    """(current device's index, stream handle) of a call; None stands for the current stream."""
    import torch
    if not torch.cuda.is_initialized():
        if not torch.cuda.is_available():
            raise ValueError("the tensors must be on a CUDA device, and there is none")
        torch.cuda.init()
    dev = torch._C._cuda_getDevice()
    if stream is None:
        return dev, torch._C._cuda_getCurrentRawStream(dev)
    if stream.device.index != dev:
        raise ValueError("stream must be one of the current CUDA device, %d (got %s)" % (dev, stream.device))
    return dev, stream.cuda_stream


def _empty(shape, dtype, stream):
    """A new tensor on the current device.  It belongs to `stream` (None: the current one), so that
    its memory is not given to another stream's work while the call's kernels use it."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device="cuda")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device="cuda")


def _is_dense(t):
    """Whether t's elements fill a block of memory in some order of its axes."""
    n = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != n:
            return False
        n *= size
    return True


def _same_order(a, b):
    """Whether two dense tensors of one shape have their elements in the same order in memory."""
    return a.is_contiguous() and b.is_contiguous() or \
        all(x == y for x, y, n in zip(a.stride(), b.stride(), a.shape) if n != 1)


def _tensor_list(tensors, what, dev, like=None):
    """The C list of CUDA tensors (dss_tensor[n]: address, count, dtype and a zero, as three 64-bit
    words each), the tensors as a list, and whether all of them are contiguous.  `like` is such a
    result for other tensors, whose types, shapes and orders of elements these have to have."""
    import torch
    T = torch.Tensor
    if isinstance(tensors, T):
        raise ValueError("%s must be a list of tensors" % what)
    codes, tensors = _dtype_codes(), list(tensors)
    n = len(tensors)
    try:
        devices = set(map(T.get_device, tensors))
    except TypeError:
        raise ValueError("%s must be a list of tensors" % what) from None
    if devices - {dev}:
        raise ValueError("%s must be on the current CUDA device, %d" % (what, dev))
    kinds = set(map(T.dtype.__get__, tensors))
    if not kinds <= codes.keys():
        raise ValueError("%s must be float32 or bfloat16 (got %s)" % (what, (kinds - codes.keys()).pop()))
    dtypes = array.array("q", [codes[k] for k in kinds] * n if len(kinds) == 1 else [codes[t.dtype] for t in tensors])
    plain = all(map(T.is_contiguous, tensors))
    if not plain and not all([t.is_contiguous() or _is_dense(t) for t in tensors]):
        raise ValueError("%s must be dense in memory, without gaps or repeated elements" % what)
    if like is None:
        counts = array.array("q", map(T.numel, tensors))
    else:
        words, others, others_plain = like
        if dtypes != words[2::3] or not all(map(T.is_same_size, tensors, others)) or not (plain and others_plain) and \
                not all(map(_same_order, tensors, others)):
            raise ValueError("%s must be of the gradients' number, types, shapes and strides" % what)
        counts = words[1::3]
    words = array.array("q", bytes(24 * n))
    words[0::3] = array.array("q", map(T.data_ptr, tensors))
    words[1::3] = counts
    words[2::3] = dtypes
    return words, tensors, plain


def grad_norm(grads, norm=None, workspace=None, stream=None):
    """The norm of a gradient over a list of CUDA tensors (float32 and bfloat16, dense in
    memory, any sizes): sqrt of the sum of all squares, as a float32 tensor of no axes."""
    dev, handle = _launch(stream)
    a, grads, _ = _tensor_list(grads, "grads", dev)
    norm, wp, wb, keep = _norm_buffers(norm, workspace, dev, stream)
    _check(lib().dss_grad_norm(a.buffer_info()[0], len(grads), norm.data_ptr(), wp, wb, handle), "dss_grad_norm")
    return norm


def clip_grads(grads, max_norm, out=None, norm=None, workspace=None, stream=None):
    """Scales a gradient, given as for grad_norm, by min(1, max_norm / (norm + 1e-6)); max_norm may be
    infinite (nothing is clipped unless the norm is NaN).
    Returns (norm, list of scaled tensors).  `out` is the list of tensors to write (allocated if
    None; `out=grads` clips in place): of the same types, shapes and strides (of axes longer than 1).
    An output shares no memory with another one (so that no tensor can be
    clipped in place twice) or with another tensor's gradient."""
    import torch
    dev, handle = _launch(stream)
    in_place = out is grads
    a, grads, plain = _tensor_list(grads, "grads", dev)
    if in_place:
        b, out = a, grads
    else:
        if out is None:
            if stream is None:
                out = [torch.empty_like(g) for g in grads]
            else:
                with torch.cuda.stream(stream):
                    out = [torch.empty_like(g) for g in grads]
        b, out, _ = _tensor_list(out, "out", dev, (a, grads, plain))
    norm, wp, wb, keep = _norm_buffers(norm, workspace, dev, stream)
    ptrs = b[0::3]
    # (an empty tensor's address is 0)
    if len(set(ptrs)) != len(ptrs) - max(ptrs.count(0) - 1, 0):
        raise ValueError("out must not have the same tensor twice")
    _check(lib().dss_clip_grads(a.buffer_info()[0], ptrs.buffer_info()[0], len(grads), max_norm, norm.data_ptr(), wp, wb,
                                handle), "dss_clip_grads")
    return norm, out


def _norm_buffers(norm, workspace, dev, stream):
    import torch
    if norm is None:
        norm = _empty((), torch.float32, stream)
    elif not isinstance(norm, torch.Tensor) or norm.dtype != torch.float32 or norm.numel() != 1 or \
            norm.get_device() != dev:
        raise ValueError("norm must be one float32 on the current CUDA device")
    if workspace is None:
        workspace = _empty(GRAD_NORM_WORKSPACE_BYTES, torch.uint8, stream)
        return norm, workspace.data_ptr(), GRAD_NORM_WORKSPACE_BYTES, workspace
    return (norm,) + _room(workspace, dev) + (workspace,)


def _room(workspace, dev):
    """(address, bytes) of a caller's workspace."""
    import torch
    if not isinstance(workspace, torch.Tensor) or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the current CUDA device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


# ---------------------------------------------------------------------------- tokens in 8 bits

_MOST = 2 ** 31 - 1      # channels and outputs: the C calls take them in 32 bits, into which ctypes would cut larger ones


def _check_tokens(x, dev):
    """dss_dtype, M, K of a matrix of tokens."""
    import torch
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a tensor [tokens][channels]")
    dt = _dtype_codes().get(x.dtype)
    if dt is None:
        raise ValueError("x must be float32 or bfloat16 (got %s)" % x.dtype)
    if x.get_device() != dev:
        raise ValueError("x must be on the current CUDA device (got %s)" % x.device)
    M, K = x.shape
    if K > _MOST:
        raise ValueError("x has %d channels, more than %d" % (K, _MOST))
    return dt, M, K


def _check_vector(t, what, n, dev):
    """The address of n float32 values."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != n or \
            not t.is_contiguous() or t.get_device() != dev:
        raise ValueError("%s must be a contiguous float32 tensor of %d elements on the current CUDA device" % (what, n))
    return t.data_ptr()


def _check_codes(t, what, rows, channels, dev):
    """(address, row stride) of a matrix of codes; one row alone may have any stride."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int8 or t.dim() != 2 or t.get_device() != dev:
        raise ValueError("%s must be an int8 matrix on the current CUDA device" % what)
    m, k = t.shape
    if rows is not None and m != rows or channels is not None and k != channels:
        raise ValueError("%s must be [%s][%s] (got [%d][%d])" % (what, "any" if rows is None else rows,
                                                                 "any" if channels is None else channels, m, k))
    rs, cs = t.stride()
    if k > 1 and cs != 1 or m > 1 and rs < k:
        raise ValueError("%s must have adjacent channels and rows that do not overlap" % what)
    return t.data_ptr(), rs if m > 1 else max(rs, k)


def quantize_tokens(x, codes=None, scales=None, stream=None):
    """8-bit codes and scales of the tokens (rows) of x, a float32 or bfloat16 CUDA matrix
    [M][K] whose channels (x.stride(1) == 1) or tokens (x.stride(0) == 1, as for
    `eval_dense(...).flatten(1).t()`) are adjacent:
      scale = max|row| / 127,  code = round(row / scale) clamped to -127 .. 127 (ties to even).
    Returns (codes int8 [M][K], scales float32 [M]).  A weight matrix [N][K] is coded the
    same way, with a scale for each output channel."""
    import torch
    dev, handle = _launch(stream)
    dt, M, K = _check_tokens(x, dev)
    if codes is None:
        codes = _empty((M, K), torch.int8, stream)
    if scales is None:
        scales = _empty(M, torch.float32, stream)
    cp, cstride = _check_codes(codes, "codes", M, K, dev)
    sp = _check_vector(scales, "scales", M, dev)
    ts, ks = x.stride()
    _check(lib().dss_quantize_tokens(x.data_ptr(), dt, M, K, ts, ks, cp, cstride, sp, handle), "dss_quantize_tokens")
    return codes, scales


def _layer_args(M, K, weight, weight_scales, bias, act, out, out_dtype, planar, dev, stream):
    """Checks a layer's weights and output: (out, N, the C arguments from the weight to the output's strides)."""
    import torch
    wp, wstride = _check_codes(weight, "weight", None, K, dev)
    N = weight.shape[0]
    if N > _MOST:
        raise ValueError("weight has %d outputs, more than %d" % (N, _MOST))
    sp = _check_vector(weight_scales, "weight_scales", N, dev)
    bp = None if bias is None else _check_vector(bias, "bias", N, dev)
    if act not in ACTS:
        raise ValueError("unknown activation %r" % (act,))
    codes, shape = _dtype_codes(), (N, M) if planar else (M, N)
    if out is None:
        out_dtype = out_dtype or torch.float32
        if out_dtype not in codes:
            raise ValueError("out_dtype must be float32 or bfloat16 (got %s)" % out_dtype)
        out = _empty(shape, out_dtype, stream)
    elif not isinstance(out, torch.Tensor) or out.shape != shape or out.dtype not in codes or out.get_device() != dev:
        raise ValueError("out must be a float32 or bfloat16 tensor of shape %s on the current CUDA device" % (shape,))
    elif out_dtype is not None and out.dtype != out_dtype:
        raise ValueError("out is %s, not out_dtype %s" % (out.dtype, out_dtype))
    s0, s1 = out.stride()
    return out, N, (wp, wstride, sp, N, K, bp, ACTS[act], out.data_ptr(), codes[out.dtype]) + \
        ((s1, s0) if planar else (s0, s1))


def _tokens_room(M, N, K, source, workspace, dev, stream):
    """(address, bytes) of a call's workspace, and what keeps it.  source: dss_token_source."""
    import torch
    if workspace is not None:
        return _room(workspace, dev) + (workspace,)
    need = ctypes.c_int64()
    _check(lib().dss_tokens_workspace(M, N, K, source, need), "dss_tokens_workspace")
    if need.value == 0:
        return None, 0, None
    workspace = _empty(need.value, torch.uint8, stream)
    return workspace.data_ptr(), need.value, workspace


def matmul_i8(codes, scales, weight, weight_scales, bias=None, act="none", out=None, out_dtype=None, planar=False,
              workspace=None, stream=None):
    """A fully connected layer on tokens in 8 bits (quantize_tokens' codes [M][K] and scales [M])
    with weights in 8 bits (codes [N][K], scales [N]):
      y[m][n] = act(scales[m] * weight_scales[n] * sum_k codes[m][k] * weight[n][k] + bias[n]),
    the sum exact.  act is "none", "relu" or "tanh".  Returns out, [M][N] or with planar=True the
    dense map [N][M], of out_dtype (float32, or `out`'s, unless given); an `out` of any row stride is
    taken."""
    dev, handle = _launch(stream)
    cp, cstride = _check_codes(codes, "codes", None, None, dev)
    M, K = codes.shape
    if K > _MOST:
        raise ValueError("codes have %d channels, more than %d" % (K, _MOST))
    sp = _check_vector(scales, "scales", M, dev)
    out, N, args = _layer_args(M, K, weight, weight_scales, bias, act, out, out_dtype, planar, dev, stream)
    room, size, keep = _tokens_room(M, N, K, 2, workspace, dev, stream)
    _check(lib().dss_matmul_tokens(cp, cstride, sp, M, *args, room, size, handle), "dss_matmul_tokens")
    return out


def linear_i8(x, weight, weight_scales, bias=None, act="none", out=None, out_dtype=None, planar=False,
              workspace=None, stream=None):
    """matmul_i8 on float32 or bfloat16 tokens x [M][K], given as for quantize_tokens: codes them
    and multiplies in one call, with the same bits as the two calls."""
    dev, handle = _launch(stream)
    dt, M, K = _check_tokens(x, dev)
    ts, ks = x.stride()
    out, N, args = _layer_args(M, K, weight, weight_scales, bias, act, out, out_dtype, planar, dev, stream)
    room, size, keep = _tokens_room(M, N, K, 1 if ks != 1 and K > 1 else 0, workspace, dev, stream)
    _check(lib().dss_linear_tokens(x.data_ptr(), dt, M, ts, ks, *args, room, size, handle), "dss_linear_tokens")
    return out
