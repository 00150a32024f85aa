"""The library's stateless operators on torch tensors: checks of arguments, outputs, and the call on torch's current stream.

linear_recurrence, linear_recurrence_backward    a recurrence whose gates do not see the state, over whole sequences or one step
rms_norm, rms_norm_fp8, rms_norm_backward        the norm of rows, with the residual's addition
fp8_quantize, fp8_product                        8-bit matrices with a scale for each 128 columns, and their product

Tensors are CUDA tensors of one device; activations are bf16 or fp32 (all of a call of one type), states, scales, norm weights
and biases fp32.  Only the last dimension has to be contiguous, unless said otherwise.  Every call enqueues kernels on torch's
current stream of that device and returns; outputs are new tensors unless an ``out`` is taken, which may share no element with
an input.  Calls that cannot be served raise ValueError (the tensors) or LstmError (what the library refused).  The calls record no graph: gradients are calls of their own, and
while torch records gradients, tensors that require them are refused.

A step of generation makes a few of these calls, each of a few microseconds on the GPU, so the checks here are few and plain.
"""
from __future__ import annotations

import ctypes
import math
import threading

import numpy as np
import torch

from . import binding as _b
from .binding import LSTM_LINREC_GATE, LSTM_LINREC_REVERSE, LSTM_LINREC_SEGMENT, LstmError

_TYPES = {torch.bfloat16: _b.LSTM_BF16, torch.float32: _b.LSTM_F32}
_F32, _I32, _E4M3 = torch.float32, torch.int32, torch.float8_e4m3fn
_empty = torch.empty
_reason = threading.local()
_functions = {}


def _function(name):
    fn = _functions.get(name)
    if fn is None:
        fn = _functions[name] = getattr(_b.load_library(), name)
    return fn


def _call(name, device, *args):
    """The C function of that name on ``device`` (its index) and torch's current stream there."""
    try:
        err = _reason.buffer
    except AttributeError:
        err = _reason.buffer = ctypes.create_string_buffer(160)
    before = _current_device()
    if before == device:
        rc = _function(name)(*args, _stream(device), err, 160)
    else:
        torch.cuda.set_device(device)
        try:
            rc = _function(name)(*args, _stream(device), err, 160)
        finally:
            torch.cuda.set_device(before)
    if rc:
        raise LstmError(rc, err.value.decode())


def _stream_of(device):
    return torch.cuda.current_stream(device).cuda_stream


# the same numbers without objects and checks around them, where this torch has them (the tensors have initialised CUDA)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_of)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


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
    """The address and the strides of a tensor that is as the call needs it, else ValueError."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == device:
            strides = t.stride()
            if strides[-1] == 1 or shape[-1] < 2:
                return t.data_ptr(), strides
    except AttributeError:
        raise ValueError(f"{name} must be a CUDA tensor") from None
    raise ValueError(f"{name} must be {dtype} {tuple(shape)} on cuda:{device} with a contiguous last dimension, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _whole(t, name, shape, dtype, device):
    """The address of a contiguous tensor; 0 for None."""
    if t is None:
        return 0
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        raise ValueError(f"{name} must be a CUDA tensor") from None
    raise ValueError(f"{name} must be contiguous {dtype} {tuple(shape)} on cuda:{device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


_recording = torch.is_grad_enabled


def _no_graph():
    """No gradient is lost without a word."""
    raise ValueError("this call records no graph for a tensor that requires gradients: call it under torch.no_grad() or detach the tensor "
                     "(linear_recurrence_backward and rms_norm_backward compute gradients)")


# the library counts in 32 bits, and ctypes would cut off what is above
_MOST = 0x7fffffff


def _too_large():
    raise ValueError("dimensions of 2^31 and more are not served")


def _apart(t, name):
    """Outputs that are written: no two elements of them may be one."""
    reach = t.shape[-1] if t.dim() else 0
    for stride, size in sorted((t.stride(d), t.shape[d]) for d in range(t.dim() - 1) if t.shape[d] > 1):
        if stride < reach:
            raise ValueError(f"{name}: elements of an output may not share memory")
        reach += stride * (size - 1)


def _runs(t):
    """The addresses at which a tensor's runs of contiguous elements begin, in order, and their bytes."""
    es, starts = t.element_size(), np.zeros(1, dtype=np.int64)
    for size, stride in zip(t.shape[:-1], t.stride()[:-1]):
        starts = (starts[:, None] + np.arange(size if stride else 1, dtype=np.int64) * (stride * es)).reshape(-1)
    return np.sort(starts) + t.data_ptr(), t.shape[-1] * es


def _share(out, t):
    """Is an element of ``out`` (none of which overlap) also one of ``t``?"""
    run, other = out.shape[-1] * out.element_size(), t.shape[-1] * t.element_size()
    # runs at a common distance, those of one beside those of the other (halves of one matrix)
    pitch = math.gcd(*(st * v.element_size() for v in (out, t) for st, n in zip(v.stride()[:-1], v.shape) if n > 1))
    if pitch:
        at = (out.data_ptr() - t.data_ptr()) % pitch
        if at >= other and at + run <= pitch:
            return False
    begin, run = _runs(out)
    theirs, other = _runs(t)
    last = np.searchsorted(begin, theirs + other) - 1              # the last of out's runs that begins in front of the end of each
    return bool(((last >= 0) & (begin[last] + run > theirs)).any())


def _no_input(out, name, *inputs):
    """``out`` shares no element with the inputs (tensors or None, each with its name)."""
    if not out.numel():
        return
    at, end = _range(out)
    for t, other in inputs:
        if t is not None and t.numel():
            begin, stop = _range(t)
            if begin < end and at < stop and _share(out, t):
                raise ValueError(f"{name} overlaps {other}")


def _range(t):
    at = t.data_ptr()
    return at, at + (sum([(n - 1) * st for n, st in zip(t.shape, t.stride())]) + 1) * t.element_size()


# ---------------------------------------------------------------- recurrence
def _workspace(T, B, D, device):
    """A call's workspace, or None.  It is held until the call has been enqueued; torch's allocator orders its next use behind that."""
    need = _function("lstm_linear_recurrence_workspace")(T, B, D)
    return _empty((need,), dtype=_F32, device=device) if need > 0 else None


def linear_recurrence(a, x, h0=None, lengths=None, *, gate=True, reverse=False, save=False, out=None, state=None):
    """h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(a), or (``gate`` false) h_t = a_t h_{t-1} + x_t.

    a, x: [T, B, D]; h0: fp32 [B, D] or None (zeros); lengths: int32 [B] on the device or None; ``reverse``: every sequence from its
    last step to its first.  Returns (h, hT, states): h [T, B, D] (zero behind a sequence's end), hT fp32 [B, D] the state behind
    the last step, states fp32 [ceil(T / 16), B, D] for the backward pass with ``save``, else None.  ``out``: a tensor for h;
    ``state``: a contiguous one for hT, which may be h0 itself (a step of generation updates its state in place) but no part of
    another tensor of the call."""
    dev, dt = _first(a, "a")
    shape, dtype, device = a.shape, a.dtype, a.device
    T, B, D = shape
    if T > _MOST or B > _MOST or D > _MOST:
        _too_large()
    rows = (B, D)
    pa, (a_t, a_b, _) = _ptr(a, "a", shape, dtype, dev)
    px, (x_t, x_b, _) = _ptr(x, "x", shape, dtype, dev)
    out_given, state_given = out is not None, state is not None
    if out is None:
        out = _empty(shape, dtype=dtype, device=device)
        po, o_t, o_b = out.data_ptr(), B * D, D
    else:
        po, (o_t, o_b, _) = _ptr(out, "out", shape, dtype, dev)
        _apart(out, "out")
    if state is None:
        state = _empty(rows, dtype=_F32, device=device)
        ps = state.data_ptr()
    else:
        ps = _whole(state, "state", rows, _F32, dev)
    ph = 0 if h0 is None else ps if h0 is state else _whole(h0, "h0", rows, _F32, dev)
    pl = 0 if lengths is None else _whole(lengths, "lengths", (B,), _I32, dev)
    if out_given or state_given:            # ranges of addresses first; only where two meet does it matter which elements lie in them
        es, n, m = 2 if dt == _b.LSTM_BF16 else 4, 4 * B * D, 4 * B
        ea = pa + es * ((T - 1) * a_t + (B - 1) * a_b + D)
        ex = px + es * ((T - 1) * x_t + (B - 1) * x_b + D)
        eo = po + es * ((T - 1) * o_t + (B - 1) * o_b + D)
        if out_given and (pa < eo and po < ea or px < eo and po < ex or ph < eo and po < ph + n or pl < eo and po < pl + m or ps < eo and po < ps + n):
            _no_input(out, "out", (a, "a"), (x, "x"), (h0, "h0"), (lengths, "lengths"), (state, "state"))
        end = ps + n
        if state_given and (pa < end and ps < ea or px < end and ps < ex or ph != ps and ph < end and ps < ph + n or pl < end and ps < pl + m):
            _no_input(state, "state", (a, "a"), (x, "x"), (None if ph == ps else h0, "h0"), (lengths, "lengths"))
    if _recording() and (a.requires_grad or x.requires_grad or h0 is not None and h0.requires_grad or out.requires_grad or state.requires_grad):
        _no_graph()
    states = _empty((-(-T // LSTM_LINREC_SEGMENT), B, D), dtype=_F32, device=device) if save else None
    work = _workspace(T, B, D, device) if T > 64 else None
    _call("lstm_linear_recurrence", dev, pa, a_t, a_b, px, x_t, x_b, ph, pl, T, B, D, dt,
          (LSTM_LINREC_GATE if gate else 0) | (LSTM_LINREC_REVERSE if reverse else 0), po, o_t, o_b, ps, 0 if states is None else states.data_ptr(),
          0 if work is None else work.data_ptr(), 0 if work is None else work.numel())
    return out, state, states


def linear_recurrence_backward(a, x, states, dh, dhT=None, lengths=None, *, gate=True, reverse=False):
    """Gradients of linear_recurrence from its inputs, the ``states`` that it saved, dh [T, B, D] and dhT fp32 [B, D] (or None):
    (da, dx, dh0), da and dx like a, dh0 fp32 [B, D]."""
    dev, dt = _first(a, "a")
    shape, dtype, device = a.shape, a.dtype, a.device
    T, B, D = shape
    if T > _MOST or B > _MOST or D > _MOST:
        _too_large()
    rows = (B, D)
    pa, (a_t, a_b, _) = _ptr(a, "a", shape, dtype, dev)
    px, (x_t, x_b, _) = _ptr(x, "x", shape, dtype, dev)
    pd, (d_t, d_b, _) = _ptr(dh, "dh", shape, dtype, dev)
    if states is None:
        raise ValueError("states must be those that linear_recurrence saved")
    ph, pl = _whole(dhT, "dhT", rows, _F32, dev), _whole(lengths, "lengths", (B,), _I32, dev)
    if _recording() and (a.requires_grad or x.requires_grad or dh.requires_grad or dhT is not None and dhT.requires_grad):
        _no_graph()
    da, dx = _empty(shape, dtype=dtype, device=device), _empty(shape, dtype=dtype, device=device)
    dh0 = _empty(rows, dtype=_F32, device=device)
    work = _workspace(T, B, D, device) if T > 64 else None
    _call("lstm_linear_recurrence_backward", dev, pa, a_t, a_b, px, x_t, x_b, _whole(states, "states", (-(-T // LSTM_LINREC_SEGMENT), B, D), _F32, dev),
          pd, d_t, d_b, ph, pl, T, B, D, dt,
          (LSTM_LINREC_GATE if gate else 0) | (LSTM_LINREC_REVERSE if reverse else 0), da.data_ptr(), B * D, D, dx.data_ptr(), B * D, D, dh0.data_ptr(),
          0 if work is None else work.data_ptr(), 0 if work is None else work.numel())
    return da, dx, dh0


# ---------------------------------------------------------------- norm
def _matrix(x, name):
    dev, dt = _first(x, name)
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be a matrix")
    if shape[0] > _MOST or shape[1] > _MOST:
        _too_large()
    px, (ld, _) = _ptr(x, name, shape, x.dtype, dev)
    return dev, dt, shape, px, ld


def _norm(dev, dt, shape, px, x_ld, x, weight, residual, eps, y, y_ld, scales):
    rows, width = shape
    if residual is None:
        r, pr, pres, res_ld = None, 0, 0, 0
    else:
        pres, (res_ld, _) = _ptr(residual, "residual", shape, x.dtype, dev)
        r = _empty(shape, dtype=x.dtype, device=x.device)
        pr = r.data_ptr()
    if weight is None:
        raise ValueError("weight must be a CUDA tensor")
    pw = _whole(weight, "weight", (width,), _F32, dev)
    if _recording() and (x.requires_grad or weight.requires_grad or residual is not None and residual.requires_grad):
        _no_graph()
    _call("lstm_rms_norm", dev, px, x_ld, pres, res_ld, pw, eps, rows, width, dt, y.data_ptr(), y_ld, scales, pr, width)
    return r


def rms_norm(x, weight, residual=None, *, eps=1e-6):
    """r = x + residual (x without one), y = r / sqrt(mean(r^2) + eps) * weight over the rows of x [rows, width].
    Returns (y, r), both of x's type; r is None without a residual."""
    dev, dt, shape, px, ld = _matrix(x, "x")
    y = _empty(shape, dtype=x.dtype, device=x.device)
    return y, _norm(dev, dt, shape, px, ld, x, weight, residual, eps, y, shape[1], 0)


def rms_norm_fp8(x, weight, residual=None, *, eps=1e-6):
    """rms_norm whose y is held in 8 bits, as fp8_product takes it: (q, scales, r), q float8_e4m3fn [rows, width] with rows a multiple
    of 16 bytes apart, scales fp32 [rows, ceil(width / 128)]."""
    dev, dt, shape, px, x_ld = _matrix(x, "x")
    rows, width = shape
    ld = (width + 15) // 16 * 16
    held = _empty((rows, ld), dtype=_E4M3, device=x.device)
    scales = _empty((rows, (width + 127) // 128), dtype=_F32, device=x.device)
    r = _norm(dev, dt, shape, px, x_ld, x, weight, residual, eps, held, ld, scales.data_ptr())
    return held if ld == width else held[:, :width], scales, r


def _norm_workspace(dev, rows, width):
    if _current_device() == dev:
        return max(_function("lstm_rms_norm_workspace")(rows, width), 0)
    with torch.cuda.device(dev):
        return max(_function("lstm_rms_norm_workspace")(rows, width), 0)


def rms_norm_backward(dy, r, weight, dr=None, *, eps=1e-6):
    """Gradients of rms_norm at r (x where there was no residual): dy and dr (what reaches r past the norm, or None) like r.
    Returns (dx, dw): dx, of x and of the residual alike, of r's type, dw fp32 [width]."""
    dev, dt, shape, pr, r_ld = _matrix(r, "r")
    rows, width = shape
    py, (y_ld, _) = _ptr(dy, "dy", shape, r.dtype, dev)
    pd, d_ld = 0, 0
    if dr is not None:
        pd, (d_ld, _) = _ptr(dr, "dr", shape, r.dtype, dev)
    if weight is None:
        raise ValueError("weight must be a CUDA tensor")
    pw = _whole(weight, "weight", (width,), _F32, dev)
    if _recording() and (dy.requires_grad or r.requires_grad or weight.requires_grad or dr is not None and dr.requires_grad):
        _no_graph()
    dx = _empty(shape, dtype=r.dtype, device=r.device)
    dw = _empty((width,), dtype=_F32, device=r.device)
    need = _norm_workspace(dev, rows, width)
    work = _empty((need,), dtype=_F32, device=r.device)
    _call("lstm_rms_norm_backward", dev, py, y_ld, pr, r_ld, pw, pd, d_ld, eps, rows, width, dt, dx.data_ptr(), width, dw.data_ptr(), work.data_ptr(), need)
    return dx, dw


# ---------------------------------------------------------------- 8-bit matrices
def fp8_quantize(x, *, block_rows=1):
    """x [rows, width] as (q, scales) with x ~ scale * q: a scale for each 128 columns of a row (``block_rows`` 1: activations,
    scales [rows, ceil(width / 128)]) or for each 128 x 128 block (128: weights, scales [ceil(rows / 128), ceil(width / 128)])."""
    dev, dt, (rows, width), px, x_ld = _matrix(x, "x")
    if _recording() and x.requires_grad:
        _no_graph()
    ld = (width + 15) // 16 * 16
    held = _empty((rows, ld), dtype=_E4M3, device=x.device)
    scales = _empty(((rows + block_rows - 1) // block_rows if block_rows > 0 else 0, (width + 127) // 128), dtype=_F32, device=x.device)
    _call("lstm_fp8_quantize", dev, px, x_ld, rows, width, dt, block_rows, held.data_ptr(), ld, scales.data_ptr())
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
    if rows > _MOST or outs > _MOST or width > _MOST:
        _too_large()
    dt = _TYPES.get(dtype)
    if dt is None:
        raise ValueError(f"dtype must be bf16 or fp32, got {dtype}")
    if sx is None or sw is None:
        raise ValueError("sx and sw must be CUDA tensors")
    blocks = (width + 127) // 128
    px, (x_ld, _) = _ptr(qx, "qx", (rows, width), _E4M3, dev)
    pw, (w_ld, _) = _ptr(qw, "qw", (outs, width), _E4M3, dev)
    ps, pt, pb = _whole(sx, "sx", (rows, blocks), _F32, dev), _whole(sw, "sw", ((outs + 127) // 128, blocks), _F32, dev), _whole(bias, "bias", (outs,), _F32, dev)
    if out is None:
        out = _empty((rows, outs), dtype=dtype, device=qx.device)
        po, o_ld = out.data_ptr(), outs
    else:
        po, (o_ld, _) = _ptr(out, "out", (rows, outs), dtype, dev)
        _apart(out, "out")
        end = po + (2 if dt == _b.LSTM_BF16 else 4) * ((rows - 1) * o_ld + outs)
        if (px < end and po < px + (rows - 1) * x_ld + width or pw < end and po < pw + (outs - 1) * w_ld + width or pb < end and po < pb + 4 * outs or
                ps < end and po < ps + 4 * rows * blocks or pt < end and po < pt + 4 * blocks * ((outs + 127) // 128)):
            _no_input(out, "out", (qx, "qx"), (sx, "sx"), (qw, "qw"), (sw, "sw"), (bias, "bias"))
    if _recording() and (sx.requires_grad or sw.requires_grad or bias is not None and bias.requires_grad or out.requires_grad):
        _no_graph()
    one = (width + 15) // 16 * 16           # a single row is any distance from the next
    _call("lstm_fp8_product", dev, px, x_ld if rows > 1 else one, ps, pw, w_ld if outs > 1 else one, pt, pb, rows, outs, width, dt, po, o_ld)
    return out
