"""The library's stateless operators on torch tensors: checks of arguments, outputs, and the call on torch's current stream.

linear_recurrence, linear_recurrence_backward    a recurrence whose gates do not see the state, over whole sequences or one step
rms_norm, rms_norm_fp8, rms_norm_backward        the norm of rows, with the residual's addition
fp8_quantize, fp8_product                        8-bit matrices with a scale for each 128 columns, and their product

Tensors are CUDA tensors of one device; activations are bf16 or fp32 (all of a call of one type), states, scales, norm weights
and biases fp32.  Only the last dimension has to be contiguous, unless said otherwise.  Every call enqueues kernels on torch's
current stream of that device and returns; outputs are new tensors unless an ``out`` is taken.  Calls that cannot be served raise
ValueError (the tensors) or LstmError (what the library refused).

A step of generation makes a few of these calls, each of a few microseconds on the GPU, so the checks here are few and plain.
"""
from __future__ import annotations

import ctypes
import threading

import torch

from . import binding as _b
from .binding import LSTM_LINREC_GATE, LSTM_LINREC_REVERSE, LSTM_LINREC_SEGMENT, LstmError

_TYPES = {torch.bfloat16: _b.LSTM_BF16, torch.float32: _b.LSTM_F32}
_F32, _I32, _E4M3 = torch.float32, torch.int32, torch.float8_e4m3fn
_reason = threading.local()


def _call(name, device, *args):
    """The C function of that name on ``device`` (its index) and torch's current stream there."""
    try:
        err = _reason.buffer
    except AttributeError:
        err = _reason.buffer = ctypes.create_string_buffer(160)
    fn = getattr(_b._lib or _b.load_library(), name)
    before = torch.cuda.current_device()
    if before == device:
        rc = fn(*args, _stream(device), err, 160)
    else:
        torch.cuda.set_device(device)
        try:
            rc = fn(*args, _stream(device), err, 160)
        finally:
            torch.cuda.set_device(before)
    if rc:
        raise LstmError(rc, err.value.decode())


def _stream_of(device):
    return torch.cuda.current_stream(device).cuda_stream


# the same number without an object around it, where this torch has it
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_of)


def _first(t, name):
    """Device index and type of a call from its first tensor."""
    try:
        device = t.get_device()
        dt = _TYPES.get(t.dtype)
    except AttributeError:
        raise ValueError(f"{name} must be a CUDA tensor") from None
    if device < 0:
        raise ValueError("the library works on CUDA tensors")
    if dt is None:
        raise ValueError(f"{name} must be bf16 or fp32, got {t.dtype}")
    return device, dt


def _ptr(t, name, shape, dtype, device):
    """The address of a tensor that is as the call needs it, else ValueError."""
    try:
        if t.dtype is dtype and t.get_device() == device and t.shape == shape and (t.stride(-1) == 1 or t.shape[-1] < 2):
            return t.data_ptr()
    except AttributeError:
        raise ValueError(f"{name} must be a CUDA tensor") from None
    raise ValueError(f"{name} must be {dtype} {tuple(shape)} on cuda:{device} with a contiguous last dimension, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _whole(t, name, shape, dtype, device):
    """... of a contiguous tensor; 0 for None."""
    if t is None:
        return 0
    p = _ptr(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return p


def _apart(t, name):
    """Outputs that are written: no two elements of them may be one."""
    for d in range(t.dim() - 1):
        if t.shape[d] > 1 and t.stride(d) < t.shape[-1]:
            raise ValueError(f"{name}: elements of an output may not share memory")


# ---------------------------------------------------------------- recurrence
def _workspace(T, B, D, like):
    """A call's workspace, or None.  It is held until the call has been enqueued; torch's allocator orders its next use behind that."""
    need = _b.lstm_linear_recurrence_workspace(T, B, D) if T > 64 else 0
    return torch.empty((need,), dtype=_F32, device=like.device) if need > 0 else None


def linear_recurrence(a, x, h0=None, lengths=None, *, gate=True, reverse=False, save=False, out=None, state=None):
    """h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(a), or (``gate`` false) h_t = a_t h_{t-1} + x_t.

    a, x: [T, B, D]; h0: fp32 [B, D] or None (zeros); lengths: int32 [B] on the device or None; ``reverse``: every sequence from its
    last step to its first.  Returns (h, hT, states): h [T, B, D] (zero behind a sequence's end), hT fp32 [B, D] the state behind
    the last step, states fp32 [ceil(T / 16), B, D] for the backward pass with ``save``, else None.  ``out``: a tensor for h;
    ``state``: a contiguous one for hT, which may be h0 itself (a step of generation updates its state in place)."""
    dev, dt = _first(a, "a")
    shape, dtype = a.shape, a.dtype
    T, B, D = shape
    rows = (B, D)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=a.device)
    else:
        _apart(out, "out")
    if state is None:
        state = torch.empty(rows, dtype=_F32, device=a.device)
    states = torch.empty((-(-T // LSTM_LINREC_SEGMENT), B, D), dtype=_F32, device=a.device) if save else None
    work = _workspace(T, B, D, a)
    a_t, a_b, _ = a.stride()
    px = _ptr(x, "x", shape, dtype, dev)
    x_t, x_b, _ = x.stride()
    po = _ptr(out, "out", shape, dtype, dev)
    o_t, o_b, _ = out.stride()
    _call("lstm_linear_recurrence", dev, _ptr(a, "a", shape, dtype, dev), a_t, a_b, px, x_t, x_b, _whole(h0, "h0", rows, _F32, dev),
          _whole(lengths, "lengths", (B,), _I32, dev), T, B, D, dt, (LSTM_LINREC_GATE if gate else 0) | (LSTM_LINREC_REVERSE if reverse else 0),
          po, o_t, o_b, _whole(state, "state", rows, _F32, dev), 0 if states is None else states.data_ptr(), 0 if work is None else work.data_ptr(),
          0 if work is None else work.numel())
    return out, state, states


def linear_recurrence_backward(a, x, states, dh, dhT=None, lengths=None, *, gate=True, reverse=False):
    """Gradients of linear_recurrence from its inputs, the ``states`` that it saved, dh [T, B, D] and dhT fp32 [B, D] (or None):
    (da, dx, dh0), da and dx like a, dh0 fp32 [B, D]."""
    dev, dt = _first(a, "a")
    shape, dtype = a.shape, a.dtype
    T, B, D = shape
    rows = (B, D)
    da, dx = torch.empty(shape, dtype=dtype, device=a.device), torch.empty(shape, dtype=dtype, device=a.device)
    dh0 = torch.empty(rows, dtype=_F32, device=a.device)
    work = _workspace(T, B, D, a)
    px, pd = _ptr(x, "x", shape, dtype, dev), _ptr(dh, "dh", shape, dtype, dev)
    if states is None:
        raise ValueError("states must be those that linear_recurrence saved")
    _call("lstm_linear_recurrence_backward", dev, _ptr(a, "a", shape, dtype, dev), a.stride(0), a.stride(1), px, x.stride(0), x.stride(1),
          _whole(states, "states", (-(-T // LSTM_LINREC_SEGMENT), B, D), _F32, dev), pd, dh.stride(0), dh.stride(1), _whole(dhT, "dhT", rows, _F32, dev),
          _whole(lengths, "lengths", (B,), _I32, dev), T, B, D, dt, (LSTM_LINREC_GATE if gate else 0) | (LSTM_LINREC_REVERSE if reverse else 0),
          da.data_ptr(), B * D, D, dx.data_ptr(), B * D, D, dh0.data_ptr(), 0 if work is None else work.data_ptr(),
          0 if work is None else work.numel())
    return da, dx, dh0


# ---------------------------------------------------------------- norm
def _norm(x, weight, residual, eps, y, y_ld, scales):
    dev, dt = _first(x, "x")
    shape = x.shape
    rows, width = shape
    if residual is None:
        r, pr, pres, res_ld = None, 0, 0, 0
    else:
        pres, res_ld = _ptr(residual, "residual", shape, x.dtype, dev), residual.stride(0)
        r = torch.empty(shape, dtype=x.dtype, device=x.device)
        pr = r.data_ptr()
    if weight is None:
        raise ValueError("weight must be a CUDA tensor")
    _call("lstm_rms_norm", dev, _ptr(x, "x", shape, x.dtype, dev), x.stride(0), pres, res_ld, _whole(weight, "weight", (width,), _F32, dev), eps, rows,
          width, dt, y.data_ptr(), y_ld, 0 if scales is None else scales.data_ptr(), pr, width)
    return r


def rms_norm(x, weight, residual=None, *, eps=1e-6):
    """r = x + residual (x without one), y = r / sqrt(mean(r^2) + eps) * weight over the rows of x [rows, width].
    Returns (y, r), both of x's type; r is None without a residual."""
    _first(x, "x")
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    return y, _norm(x, weight, residual, eps, y, x.shape[1], None)


def rms_norm_fp8(x, weight, residual=None, *, eps=1e-6):
    """rms_norm whose y is held in 8 bits, as fp8_product takes it: (q, scales, r), q float8_e4m3fn [rows, width] with rows a multiple
    of 16 bytes apart, scales fp32 [rows, ceil(width / 128)]."""
    _first(x, "x")
    rows, width = x.shape
    ld = (width + 15) // 16 * 16
    held = torch.empty((rows, ld), dtype=_E4M3, device=x.device)
    scales = torch.empty((rows, (width + 127) // 128), dtype=_F32, device=x.device)
    r = _norm(x, weight, residual, eps, held, ld, scales)
    return held if ld == width else held[:, :width], scales, r


def rms_norm_backward(dy, r, weight, dr=None, *, eps=1e-6):
    """Gradients of rms_norm at r (x where there was no residual): dy and dr (what reaches r past the norm, or None) like r.
    Returns (dx, dw): dx, of x and of the residual alike, of r's type, dw fp32 [width]."""
    dev, dt = _first(r, "r")
    shape, dtype = r.shape, r.dtype
    rows, width = shape
    dx = torch.empty(shape, dtype=dtype, device=r.device)
    dw = torch.empty((width,), dtype=_F32, device=r.device)
    py = _ptr(dy, "dy", shape, dtype, dev)
    pd, d_ld = (0, 0) if dr is None else (_ptr(dr, "dr", shape, dtype, dev), dr.stride(0))
    if weight is None:
        raise ValueError("weight must be a CUDA tensor")
    with torch.cuda.device(dev):
        need = max(_b.lstm_rms_norm_workspace(rows, width), 0)
    workspace = torch.empty((need,), dtype=_F32, device=r.device)
    _call("lstm_rms_norm_backward", dev, py, dy.stride(0), _ptr(r, "r", shape, dtype, dev), r.stride(0), _whole(weight, "weight", (width,), _F32, dev),
          pd, d_ld, eps, rows, width, dt, dx.data_ptr(), width, dw.data_ptr(), workspace.data_ptr(), need)
    return dx, dw


# ---------------------------------------------------------------- 8-bit matrices
def fp8_quantize(x, *, block_rows=1):
    """x [rows, width] as (q, scales) with x ~ scale * q: a scale for each 128 columns of a row (``block_rows`` 1: activations,
    scales [rows, ceil(width / 128)]) or for each 128 x 128 block (128: weights, scales [ceil(rows / 128), ceil(width / 128)])."""
    dev, dt = _first(x, "x")
    rows, width = x.shape
    ld = (width + 15) // 16 * 16
    held = torch.empty((rows, ld), dtype=_E4M3, device=x.device)
    scales = torch.empty(((rows + block_rows - 1) // block_rows if block_rows > 0 else 0, (width + 127) // 128), dtype=_F32, device=x.device)
    _call("lstm_fp8_quantize", dev, _ptr(x, "x", x.shape, x.dtype, dev), x.stride(0), rows, width, dt, block_rows, held.data_ptr(), ld, scales.data_ptr())
    return held if ld == width else held[:, :width], scales


def fp8_product(qx, sx, qw, sw, bias=None, *, dtype=torch.bfloat16, out=None):
    """y = x w^T + bias of 8-bit matrices: qx [rows, width] with sx (block_rows 1), qw [outs, width] with sw (block_rows 128), bias
    fp32 [outs] or None; y [rows, outs] of ``dtype``.  Rows of qx and qw are a multiple of 16 bytes apart, as fp8_quantize and
    rms_norm_fp8 make them."""
    try:
        dev, (rows, width), outs = qx.get_device(), qx.shape, qw.shape[0]
    except (AttributeError, ValueError):
        raise ValueError("qx and qw must be CUDA matrices") from None
    if dev < 0:
        raise ValueError("the library works on CUDA tensors")
    dt = _TYPES.get(dtype)
    if dt is None:
        raise ValueError(f"dtype must be bf16 or fp32, got {dtype}")
    if sx is None or sw is None:
        raise ValueError("sx and sw must be CUDA tensors")
    blocks = (width + 127) // 128
    if out is None:
        out = torch.empty((rows, outs), dtype=dtype, device=qx.device)
    else:
        _apart(out, "out")
    _call("lstm_fp8_product", dev, _ptr(qx, "qx", (rows, width), _E4M3, dev), _ld(qx, rows, width), _whole(sx, "sx", (rows, blocks), _F32, dev),
          _ptr(qw, "qw", (outs, width), _E4M3, dev), _ld(qw, outs, width), _whole(sw, "sw", ((outs + 127) // 128, blocks), _F32, dev),
          _whole(bias, "bias", (outs,), _F32, dev), rows, outs, width, dt, _ptr(out, "out", (rows, outs), dtype, dev), out.stride(0))
    return out


def _ld(q, rows, width):
    """Row stride of 8-bit rows; a single row has any."""
    return q.stride(0) if rows > 1 else (width + 15) // 16 * 16
