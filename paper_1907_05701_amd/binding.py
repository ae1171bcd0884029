"""ctypes binding of libadpsgd_blstm.so: one Python function per C entry
point, same names, argument marshalling only.  Device buffers are torch
tensors (torch supplies memory and streams); every computation runs in the
library's HIP kernels.  The library must have been built
(``__graft_entry__.build()``); loading fails loudly otherwise."""

from __future__ import annotations

import ctypes
import os
import struct

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libadpsgd_blstm.so")

BLSTM_FP32 = 0
BLSTM_BF16 = 1
ADPSGD_ORDER_EQ7 = 1
ADPSGD_WRITE_PEER = 2
BLSTM_EINVAL = -1
BLSTM_EUNSUPPORTED = -2
BLSTM_EHIP = -3
HEAD_STATIC_SCRATCH_BYTES = 64 << 20   # the static head workspace (adpsgd_blstm.h)

EXPORTED = ("blstm_param_count", "blstm_workspace_bytes", "blstm_pack_params", "blstm_fwd",
            "softmax_ce_fwd_bwd", "softmax_ce_fwd_bwd_static", "blstm_bwd", "replica_grad_reduce", "adpsgd_step",
            "blstm_recurrence_ok", "blstm_last_error", "blstm_timing_begin", "blstm_timing_end",
            "ssm_workspace_bytes", "ssm_conv_fwd", "ssm_conv_bwd", "ssm_conv_step", "ssm_scan_fwd", "ssm_scan_bwd",
            "ssm_scan_step", "softmax_topk_rows", "softmax_distill_rows", "softmax_head_ws_bytes", "softmax_topk",
            "softmax_distill_fwd_bwd")
SSM_SOFTPLUS = 1
SSM_SILU = 2
SOFTMAX_MAX_TOP = 256                  # most listed classes a row (adpsgd_blstm.h)
SOFTMAX_MAX_CLASSES = 1 << 18


class Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("L", "D", "H", "P", "K", "T", "B", "precision")]


class SsmDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "B", "D", "N", "G", "W", "precision")]


class SsmScanIn(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "dt", "Bm", "Cm", "z")] +
                [(n, ctypes.c_int64) for n in ("ldx", "lddt", "ldb", "ldc", "ldz")] +
                [(n, ctypes.c_void_p) for n in ("A", "Dskip", "dt_bias", "h0", "lens")] + [("flags", ctypes.c_uint32)])


class SsmScanGrads(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("dx", "ddt", "dBm", "dCm", "dz")] +
                [(n, ctypes.c_int64) for n in ("lddx", "ldddt", "lddb", "lddc", "lddz")] +
                [(n, ctypes.c_void_p) for n in ("dA", "dDskip", "ddt_bias", "dh0")])


class SoftmaxTeacher(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("top", "idx", "rest", "labels", "weights")] +
                [("k", ctypes.c_int32)] + [(n, ctypes.c_float) for n in ("temperature", "soft", "hard")])


class KernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_double)]


class BlstmError(RuntimeError):
    def __init__(self, fn, code, msg):
        super().__init__(f"{fn} failed ({code}): {msg}")
        self.code = code


_lib = None


def lib():
    """Load the library once (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.c_void_p
        DP = ctypes.POINTER(Dims)
        S = ctypes.c_size_t
        L.blstm_param_count.argtypes = [DP]
        L.blstm_param_count.restype = ctypes.c_int64
        L.blstm_workspace_bytes.argtypes = [DP, ctypes.POINTER(S), ctypes.POINTER(S),
                                            ctypes.POINTER(S), ctypes.POINTER(S)]
        L.blstm_pack_params.argtypes = [DP, P, P, P]
        L.blstm_fwd.argtypes = [DP, P, P, P, P, P, P]
        L.softmax_ce_fwd_bwd.argtypes = [DP, P, P, P, P, ctypes.c_float, P, P, P, P, P]
        L.softmax_ce_fwd_bwd_static.argtypes = [DP, P, P, P, P, ctypes.c_float, P, P, P, P]
        L.blstm_bwd.argtypes = [DP, P, P, P, P, P, P, P]
        L.blstm_recurrence_ok.argtypes = [DP, P, P]
        L.replica_grad_reduce.argtypes = [ctypes.POINTER(P), ctypes.c_int32, ctypes.c_int64,
                                          ctypes.c_float, P, P]
        L.adpsgd_step.argtypes = [P, P, ctypes.POINTER(P), ctypes.c_int32, ctypes.c_float,
                                  ctypes.c_int64, ctypes.c_float, ctypes.c_uint32, P, P]
        L.blstm_last_error.restype = ctypes.c_char_p
        L.blstm_timing_begin.argtypes = [ctypes.c_char_p]
        L.blstm_timing_end.argtypes = [ctypes.POINTER(KernelTime), ctypes.c_int32,
                                       ctypes.POINTER(ctypes.c_int32)]
        I, I64, U, F = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_float
        SD, SG, ST = (ctypes.POINTER(c) for c in (SsmDims, SsmScanGrads, SoftmaxTeacher))
        L.ssm_workspace_bytes.argtypes = [SD] + [ctypes.POINTER(S)] * 4
        L.ssm_conv_fwd.argtypes = [SD, P, I64, P, P, P, P, P, I64, P, U, P]
        L.ssm_conv_bwd.argtypes = [SD, P, I64, P, P, P, P, P, I64, P, P, I64, P, P, P, P, U, P]
        L.ssm_conv_step.argtypes = [SD, P, I64, P, P, P, I, P, P, I64, U, P]
        # ssm_scan_in by its bytes
        L.ssm_scan_fwd.argtypes = [SD, P, P, I64, P, P, P, P]
        L.ssm_scan_bwd.argtypes = [SD, P, P, I64, P, P, SG, P, P]
        L.ssm_scan_step.argtypes = [SD, P, P, I, P, P, I64, P]
        L.softmax_topk_rows.argtypes = [P, I64, I64, I, I, I, F, P, P, P, P]
        L.softmax_distill_rows.argtypes = [P, I64, I64, I, I, ST, F, P, P, I64, P]
        L.softmax_head_ws_bytes.argtypes = [DP, ctypes.POINTER(S)]
        L.softmax_topk.argtypes = [DP, P, P, P, I, F, P, P, P, P, P]
        L.softmax_distill_fwd_bwd.argtypes = [DP, P, P, P, ST, F, P, P, P, P, P]
        for name in EXPORTED[-12:]:
            getattr(L, name).restype = ctypes.c_int
        for name in ("blstm_workspace_bytes", "blstm_pack_params", "blstm_fwd", "softmax_ce_fwd_bwd",
                     "softmax_ce_fwd_bwd_static",
                     "blstm_bwd", "replica_grad_reduce", "adpsgd_step", "blstm_timing_begin",
                     "blstm_timing_end"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def make_dims(L, D, H, P, K, T, B, precision):
    if isinstance(precision, str):
        precision = {"fp32": BLSTM_FP32, "bf16": BLSTM_BF16}[precision]
    return Dims(L, D, H, P, K, T, B, precision)


def _check(fn, rc):
    if rc != 0:
        raise BlstmError(fn, rc, lib().blstm_last_error().decode())
    return rc


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def blstm_param_count(dims: Dims) -> int:
    n = lib().blstm_param_count(ctypes.byref(dims))
    if n < 0:
        raise BlstmError("blstm_param_count", n, lib().blstm_last_error().decode())
    return n


def blstm_workspace_bytes(dims: Dims) -> dict:
    vals = [ctypes.c_size_t() for _ in range(4)]
    _check("blstm_workspace_bytes",
           lib().blstm_workspace_bytes(ctypes.byref(dims), *[ctypes.byref(v) for v in vals]))
    return dict(zip(("act_ws", "head_ws", "theta_lp", "y_top"), (v.value for v in vals)))


def blstm_pack_params(dims, theta, theta_lp, stream=None):
    return _check("blstm_pack_params", lib().blstm_pack_params(
        ctypes.byref(dims), _ptr(theta), _ptr(theta_lp), _stream(stream)))


def blstm_fwd(dims, theta, theta_lp, x, act_ws, y_top, stream=None):
    return _check("blstm_fwd", lib().blstm_fwd(
        ctypes.byref(dims), _ptr(theta), _ptr(theta_lp), _ptr(x), _ptr(act_ws), _ptr(y_top),
        _stream(stream)))


def softmax_ce_fwd_bwd(dims, theta, theta_lp, y_top, labels, loss_scale, loss, dy_top, grad,
                       head_ws, stream=None):
    return _check("softmax_ce_fwd_bwd", lib().softmax_ce_fwd_bwd(
        ctypes.byref(dims), _ptr(theta), _ptr(theta_lp), _ptr(y_top), _ptr(labels),
        ctypes.c_float(loss_scale), _ptr(loss), _ptr(dy_top), _ptr(grad), _ptr(head_ws),
        _stream(stream)))


def softmax_ce_fwd_bwd_static(dims, theta, theta_lp, y_top, labels, loss_scale, loss, dy_top, grad, stream=None):
    return _check("softmax_ce_fwd_bwd_static", lib().softmax_ce_fwd_bwd_static(
        ctypes.byref(dims), _ptr(theta), _ptr(theta_lp), _ptr(y_top), _ptr(labels),
        ctypes.c_float(loss_scale), _ptr(loss), _ptr(dy_top), _ptr(grad), _stream(stream)))


def blstm_bwd(dims, theta, theta_lp, act_ws, y_top, dy_top, grad, stream=None):
    return _check("blstm_bwd", lib().blstm_bwd(
        ctypes.byref(dims), _ptr(theta), _ptr(theta_lp), _ptr(act_ws), _ptr(y_top), _ptr(dy_top),
        _ptr(grad), _stream(stream)))


def blstm_recurrence_ok(dims, act_ws, stream=None):
    return _check("blstm_recurrence_ok", lib().blstm_recurrence_ok(ctypes.byref(dims), _ptr(act_ws),
                                                                   _stream(stream)))


def _ptr_array(tensors):
    arr = (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
    return ctypes.cast(arr, ctypes.POINTER(ctypes.c_void_p)), arr


def replica_grad_reduce(grads, scale, out, stream=None):
    ptrs, keep = _ptr_array(grads)
    n = grads[0].numel()
    return _check("replica_grad_reduce", lib().replica_grad_reduce(
        ptrs, len(grads), n, ctypes.c_float(scale), _ptr(out), _stream(stream)))


def adpsgd_step(theta, theta_peer, grads, scale, lr, flags=0, theta_lp=None, stream=None):
    ptrs, keep = _ptr_array(grads)
    return _check("adpsgd_step", lib().adpsgd_step(
        _ptr(theta), _ptr(theta_peer), ptrs, len(grads), ctypes.c_float(scale), theta.numel(),
        ctypes.c_float(lr), flags, _ptr(theta_lp), _stream(stream)))


def blstm_timing_begin(prefix: str = ""):
    return _check("blstm_timing_begin", lib().blstm_timing_begin(prefix.encode()))


def blstm_timing_end(cap: int = 64) -> dict:
    buf = (KernelTime * cap)()
    count = ctypes.c_int32()
    _check("blstm_timing_end", lib().blstm_timing_end(buf, cap, ctypes.byref(count)))
    return {buf[i].name.decode(): (buf[i].launches, buf[i].total_ms) for i in range(min(count.value, cap))}


# ------------------------------------------------------- state space operators ---
# Tensors are checked against the dims here, before their addresses are given
# to the library: a ValueError names the argument.
def _on(x):
    """The device index the call runs on, from its first tensor."""
    dev = x.get_device()
    if dev < 0:
        raise ValueError("tensors must be on the GPU")
    return dev


def _wrong(name, want, t, dev):
    return ValueError(f"{name} must be {want} on cuda:{dev}: got {t.dtype} {tuple(t.shape)} with strides {t.stride()} "
                      f"on {t.device}")


def _have(name, t, shape, dtype, dev, optional=False):
    """Address of a contiguous tensor of this shape and type (None for an optional one that is absent)."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or not t.is_contiguous():
        raise _wrong(name, f"a contiguous {dtype} tensor of shape {shape}", t, dev)
    return t.data_ptr()


def _rows(name, t, shape, dtype, dev, optional=False):
    """(address, row pitch) of a tensor [rows][W] or [T][B][W] whose last axis
    is contiguous and whose leading axes are rows at one pitch."""
    if t is None:
        if optional:
            return None, 0
        raise ValueError(f"{name} is required")
    if t.shape == shape and t.dtype == dtype and t.get_device() == dev:
        st, W = t.stride(), shape[-1]
        ld = st[-2]
        if len(shape) == 3:
            if shape[1] == 1:
                ld = st[0]
            elif shape[0] > 1 and st[0] != ld * shape[1]:
                ld = -1
        if ld < W and t.numel() == W:
            ld = W   # one row: its pitch says nothing
        if ld >= W and (st[-1] == 1 or W == 1):
            return t.data_ptr(), ld
    raise _wrong(name, f"{dtype} rows of shape {shape}, adjacent elements along the last axis and one pitch from row "
                       "to row,", t, dev)


def _call(fn, dev, stream, *args):
    """Calls fn on device `dev` (made current for the launch if it is not) and
    `stream`, by default the device's current one."""
    on = getattr(stream, "device", None)
    if on is not None and on.index != dev:   # its kernels would reach for another device's memory
        raise ValueError(f"the stream is on {on}, the tensors are on cuda:{dev}")
    if dev != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return _call(fn, dev, stream, *args)
    # the handle alone: a Stream object costs more than the launch's other arguments together
    s = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    rc = getattr(_lib or lib(), fn)(*args, s)
    return _check(fn, rc) if rc else rc


def _bytes(name, t, n, dev):
    if n == 0:
        return None
    if t is None or not t.is_contiguous() or t.get_device() != dev or t.numel() * t.element_size() < n:
        raise ValueError(f"{name} must be a contiguous buffer of at least {n} bytes on cuda:{dev}")
    p = t.data_ptr()
    if p % 16:
        raise ValueError(f"{name} must be 16-byte aligned")
    return p


def _elem(dims):
    return torch.bfloat16 if dims.precision == BLSTM_BF16 else torch.float32


def make_ssm_dims(T, B, D, N=1, G=1, W=1, precision="bf16"):
    if isinstance(precision, str):
        precision = {"fp32": BLSTM_FP32, "bf16": BLSTM_BF16}[precision]
    return SsmDims(T, B, D, N, G, W, precision)


_SSM_SIZES = ("saved", "fwd", "bwd", "conv_bwd")


def ssm_workspace_bytes(dims: SsmDims, only=_SSM_SIZES) -> dict:
    """Sizes in bytes by name; `only`: the buffers asked for (dims that one
    pass is too large for are refused where its buffer is asked for)."""
    vals = {n: ctypes.c_size_t() for n in only}
    _check("ssm_workspace_bytes", lib().ssm_workspace_bytes(
        ctypes.byref(dims), *[ctypes.byref(vals[n]) if n in vals else None for n in _SSM_SIZES]))
    return {n: v.value for n, v in vals.items()}


def _ssm_bytes(dims, name):
    """One of ssm_workspace_bytes, looked up once per dims object and values."""
    key = (dims.T, dims.B, dims.D, dims.N, dims.G, dims.W, dims.precision)
    got = dims.__dict__.get("sizes")
    if got is None or got[0] != key:
        got = dims.__dict__["sizes"] = (key, {})
    n = got[1].get(name)
    if n is None:
        n = got[1][name] = ssm_workspace_bytes(dims, (name,))[name]
    return n


def ssm_conv_fwd(dims, x, w, bias, y, lens=None, state=None, state_out=None, silu=True, stream=None):
    dev, e = _on(x), _elem(dims)
    T, B, D, W = dims.T, dims.B, dims.D, dims.W
    px, ldx = _rows("x", x, (T, B, D), e, dev)
    py, ldy = _rows("y", y, (T, B, D), e, dev)
    return _call("ssm_conv_fwd", dev, stream, ctypes.byref(dims), px, ldx,
                 _have("w", w, (D, W), torch.float32, dev), _have("bias", bias, (D,), torch.float32, dev, True),
                 _have("lens", lens, (B,), torch.int32, dev, True), _have("state", state, (B, W - 1, D), e, dev, True),
                 py, ldy, _have("state_out", state_out, (B, W - 1, D), e, dev, True), SSM_SILU if silu else 0)


def ssm_conv_bwd(dims, x, w, bias, dy, dx, dw, dbias, ws, lens=None, state=None, dstate=None, dstate_out=None,
                 silu=True, stream=None):
    dev, e, f = _on(x), _elem(dims), torch.float32
    T, B, D, W = dims.T, dims.B, dims.D, dims.W
    px, ldx = _rows("x", x, (T, B, D), e, dev)
    pdy, lddy = _rows("dy", dy, (T, B, D), e, dev)
    pdx, lddx = _rows("dx", dx, (T, B, D), e, dev)
    return _call("ssm_conv_bwd", dev, stream, ctypes.byref(dims), px, ldx, _have("w", w, (D, W), f, dev),
                 _have("bias", bias, (D,), f, dev, True), _have("lens", lens, (B,), torch.int32, dev, True),
                 _have("state", state, (B, W - 1, D), e, dev, True), pdy, lddy,
                 _have("dstate_out", dstate_out, (B, W - 1, D), e, dev, True), pdx, lddx,
                 _have("dw", dw, (D, W), f, dev), _have("dbias", dbias, (D,), f, dev, True),
                 _have("dstate", dstate, (B, W - 1, D), e, dev, True),
                 _bytes("ws", ws, _ssm_bytes(dims, "conv_bwd"), dev), SSM_SILU if silu else 0)


def _slots(state, slots, B, row, dtype, dev):
    """(state's address, its rows, slots' address); state is [rows][*row]."""
    if state is None or state.dim() != 1 + len(row):
        raise ValueError(f"state must be a tensor of rows of shape {row}")
    n = state.shape[0]
    return (_have("state", state, (n, *row), dtype, dev), n,
            _have("slots", slots, (B,), torch.int32, dev, True))


def ssm_conv_step(dims, x, w, bias, state, y, slots=None, silu=True, stream=None):
    dev, e = _on(x), _elem(dims)
    B, D, W = dims.B, dims.D, dims.W
    px, ldx = _rows("x", x, (B, D), e, dev)
    py, ldy = _rows("y", y, (B, D), e, dev)
    ps, n, psl = _slots(state, slots, B, (W - 1, D), e, dev)
    return _call("ssm_conv_step", dev, stream, ctypes.byref(dims), px, ldx, _have("w", w, (D, W), torch.float32, dev),
                 _have("bias", bias, (D,), torch.float32, dev, True), psl, n, ps, py, ldy, SSM_SILU if silu else 0)


_SCAN_IN = struct.Struct("@5P5q5PI4x")
assert _SCAN_IN.size == ctypes.sizeof(SsmScanIn)


def _scan_in(dims, lead, dev, x, dt, A, Bm, Cm, Dskip, z, dt_bias, h0, lens, softplus):
    e, f = _elem(dims), torch.float32
    B, D, N, GN = dims.B, dims.D, dims.N, dims.G * dims.N
    px, ldx = _rows("x", x, (*lead, D), e, dev)
    pdt, lddt = _rows("dt", dt, (*lead, D), e, dev)
    pb, ldb = _rows("Bm", Bm, (*lead, GN), e, dev)
    pc, ldc = _rows("Cm", Cm, (*lead, GN), e, dev)
    pz, ldz = _rows("z", z, (*lead, D), e, dev, True)
    # SsmScanIn's bytes (filling the ctypes structure field by field takes longer than the launch)
    return _SCAN_IN.pack(px, pdt, pb, pc, pz or 0, ldx, lddt, ldb, ldc, ldz, _have("A", A, (D, N), f, dev),
                         _have("Dskip", Dskip, (D,), f, dev, True) or 0,
                         _have("dt_bias", dt_bias, (D,), f, dev, True) or 0,
                         _have("h0", h0, (B, D, N), f, dev, True) or 0,
                         _have("lens", lens, (B,), torch.int32, dev, True) or 0, SSM_SOFTPLUS if softplus else 0)


def ssm_scan_fwd(dims, x, dt, A, Bm, Cm, y, ws, Dskip=None, z=None, dt_bias=None, h0=None, h_last=None, lens=None,
                 softplus=True, saved=None, stream=None):
    dev = _on(x)
    T, B, D, N = dims.T, dims.B, dims.D, dims.N
    arg = _scan_in(dims, (T, B), dev, x, dt, A, Bm, Cm, Dskip, z, dt_bias, h0, lens, softplus)
    py, ldy = _rows("y", y, (T, B, D), _elem(dims), dev)
    return _call("ssm_scan_fwd", dev, stream, ctypes.byref(dims), arg, py, ldy,
                 _have("h_last", h_last, (B, D, N), torch.float32, dev, True),
                 None if saved is None else _bytes("saved", saved, _ssm_bytes(dims, "saved"), dev),
                 _bytes("ws", ws, _ssm_bytes(dims, "fwd"), dev))


def ssm_scan_bwd(dims, x, dt, A, Bm, Cm, dy, saved, ws, dx, ddt, dA, dBm, dCm, Dskip=None, dDskip=None, z=None,
                 dz=None, dt_bias=None, ddt_bias=None, dh_last=None, dh0=None, lens=None, softplus=True, stream=None):
    dev, e, f = _on(x), _elem(dims), torch.float32
    T, B, D, N, GN = dims.T, dims.B, dims.D, dims.N, dims.G * dims.N
    arg = _scan_in(dims, (T, B), dev, x, dt, A, Bm, Cm, Dskip, z, dt_bias, None, lens, softplus)
    pdy, lddy = _rows("dy", dy, (T, B, D), e, dev)
    pdx, lddx = _rows("dx", dx, (T, B, D), e, dev)
    pdt, ldddt = _rows("ddt", ddt, (T, B, D), e, dev)
    pdb, lddb = _rows("dBm", dBm, (T, B, GN), e, dev)
    pdc, lddc = _rows("dCm", dCm, (T, B, GN), e, dev)
    pdz, lddz = _rows("dz", dz, (T, B, D), e, dev, z is None)
    out = SsmScanGrads(pdx, pdt, pdb, pdc, pdz, lddx, ldddt, lddb, lddc, lddz, _have("dA", dA, (D, N), f, dev),
                       _have("dDskip", dDskip, (D,), f, dev, True), _have("ddt_bias", ddt_bias, (D,), f, dev, True),
                       _have("dh0", dh0, (B, D, N), f, dev, True))
    return _call("ssm_scan_bwd", dev, stream, ctypes.byref(dims), arg, pdy, lddy,
                 _have("dh_last", dh_last, (B, D, N), f, dev, True), _bytes("saved", saved, _ssm_bytes(dims, "saved"), dev),
                 ctypes.byref(out), _bytes("ws", ws, _ssm_bytes(dims, "bwd"), dev))


def ssm_scan_step(dims, x, dt, A, Bm, Cm, state, y, Dskip=None, z=None, dt_bias=None, slots=None, softplus=True,
                  stream=None):
    dev = _on(x)
    B, D, N = dims.B, dims.D, dims.N
    arg = _scan_in(dims, (B,), dev, x, dt, A, Bm, Cm, Dskip, z, dt_bias, None, None, softplus)
    py, ldy = _rows("y", y, (B, D), _elem(dims), dev)
    ps, n, psl = _slots(state, slots, B, (D, N), torch.float32, dev)
    return _call("ssm_scan_step", dev, stream, ctypes.byref(dims), arg, psl, n, ps, py, ldy)


# ---------------------------------------------------------------- distillation ---
def _logits(logits):
    if logits.dim() != 2 or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"logits must be bfloat16 or float32 rows [M][K]: got {logits.dtype} {tuple(logits.shape)}")
    M, K = logits.shape
    p, ld = _rows("logits", logits, (M, K), logits.dtype, _on(logits))
    return p, ld, M, K, BLSTM_BF16 if logits.dtype == torch.bfloat16 else BLSTM_FP32


def softmax_topk_rows(logits, top, idx, rest=None, temperature=1.0, stream=None):
    """k is top's width."""
    p, ld, M, K, prec = _logits(logits)
    dev, k = logits.get_device(), top.shape[-1]
    return _call("softmax_topk_rows", dev, stream, p, ld, M, K, prec, k, temperature,
                 _have("top", top, (M, k), torch.float32, dev), _have("idx", idx, (M, k), torch.int32, dev),
                 _have("rest", rest, (M,), torch.float32, dev, True))


def _teacher(M, dev, top, idx, rest, labels, weights, temperature, soft, hard):
    k = top.shape[-1]
    return SoftmaxTeacher(_have("top", top, (M, k), torch.float32, dev), _have("idx", idx, (M, k), torch.int32, dev),
                          _have("rest", rest, (M,), torch.float32, dev, True),
                          _have("labels", labels, (M,), torch.int32, dev, True),
                          _have("weights", weights, (M,), torch.float32, dev, True), k, temperature, soft, hard)


def softmax_distill_rows(logits, top, idx, row_loss, dlogits, rest=None, labels=None, weights=None, temperature=1.0,
                         soft=1.0, hard=0.0, loss_scale=1.0, stream=None):
    p, ld, M, K, prec = _logits(logits)
    dev = logits.get_device()
    t = _teacher(M, dev, top, idx, rest, labels, weights, temperature, soft, hard)
    pd, ldd = _rows("dlogits", dlogits, (M, K), logits.dtype, dev)
    return _call("softmax_distill_rows", dev, stream, p, ld, M, K, prec, ctypes.byref(t), loss_scale,
                 _have("row_loss", row_loss, (M,), torch.float32, dev), pd, ldd)


def softmax_head_ws_bytes(dims: Dims) -> int:
    n = ctypes.c_size_t()
    _check("softmax_head_ws_bytes", lib().softmax_head_ws_bytes(ctypes.byref(dims), ctypes.byref(n)))
    return n.value


def _head_args(dims, dev, theta, theta_lp, y_top, ws):
    """Addresses of the head's inputs and workspace, whose sizes dims give."""
    key = tuple(getattr(dims, n) for n, _ in Dims._fields_)
    got = dims.__dict__.get("head")
    if got is None or got[0] != key:
        got = dims.__dict__["head"] = (key, blstm_param_count(dims), softmax_head_ws_bytes(dims))
    n, e = got[1], _elem(dims)
    return (_have("theta", theta, (n,), torch.float32, dev),
            _have("theta_lp", theta_lp, (n,), torch.bfloat16, dev) if dims.precision == BLSTM_BF16 else None,
            _have("y_top", y_top, (dims.T, dims.B, 2 * dims.H), e, dev), _bytes("ws", ws, got[2], dev))


def softmax_topk(dims, theta, theta_lp, y_top, top, idx, ws, rest=None, temperature=1.0, stream=None):
    """top, idx [T*B][k], rest [T*B]; k is top's width."""
    dev, M, k = _on(y_top), dims.T * dims.B, top.shape[-1]
    pt, pl, py, pw = _head_args(dims, dev, theta, theta_lp, y_top, ws)
    return _call("softmax_topk", dev, stream, ctypes.byref(dims), pt, pl, py, k, temperature,
                 _have("top", top, (M, k), torch.float32, dev), _have("idx", idx, (M, k), torch.int32, dev),
                 _have("rest", rest, (M,), torch.float32, dev, True), pw)


def softmax_distill_fwd_bwd(dims, theta, theta_lp, y_top, top, idx, loss_scale, loss, dy_top, grad, ws, rest=None,
                            labels=None, weights=None, temperature=1.0, soft=1.0, hard=0.0, stream=None):
    dev, M = _on(y_top), dims.T * dims.B
    pt, pl, py, pw = _head_args(dims, dev, theta, theta_lp, y_top, ws)
    t = _teacher(M, dev, top, idx, rest, labels, weights, temperature, soft, hard)
    return _call("softmax_distill_fwd_bwd", dev, stream, ctypes.byref(dims), pt, pl, py, ctypes.byref(t), loss_scale,
                 _have("loss", loss, (1,), torch.float32, dev),
                 _have("dy_top", dy_top, (dims.T, dims.B, 2 * dims.H), torch.float32, dev),
                 _have("grad", grad, tuple(theta.shape), torch.float32, dev), pw)
