"""The library's stateless operators on torch tensors: checks of arguments, outputs, and the call on torch's current stream.

linear_recurrence, linear_recurrence_backward    a recurrence whose gates do not see the state, over whole sequences or one step
rms_norm, rms_norm_fp8, rms_norm_backward        the norm of rows, with the residual's addition
fp8_quantize, fp8_product                        8-bit matrices with a scale for each 128 columns, and their product

Tensors are CUDA tensors of one device; activations are bf16 or fp32 (all of a call of one type), states, scales, norm weights
and biases fp32.  Only the last dimension has to be contiguous, unless said otherwise.  Every call enqueues kernels on torch's
current stream of that device and returns; outputs are new tensors unless an ``out`` is taken.  Calls that cannot be served raise
ValueError (the tensors) or LstmError (what the library refused).
"""
from __future__ import annotations

import torch

from . import binding as _b
from .binding import LSTM_LINREC_GATE, LSTM_LINREC_REVERSE, LSTM_LINREC_SEGMENT, LstmError

_TYPES = {torch.bfloat16: _b.LSTM_BF16, torch.float32: _b.LSTM_F32}


def _check(result):
    if result[0]:
        raise LstmError(*result)


def _device(t):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("the library works on CUDA tensors")
    return t.device


def _want(t, name, shape, dtype, device, contiguous=False, optional=False):
    """The address of t if it is as the call needs it, else ValueError; 0 for an optional one that is None."""
    if t is None and optional:
        return 0
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype or t.device != device or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr()


def _type(t, name):
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be bf16 or fp32, got {t.dtype}")
    return code


class _On:
    """The current device for the length of a call, changed only where it is another one."""

    def __init__(self, device):
        self.index = device.index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *_):
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def _own_steps(t, name):
    """Outputs that are written: no two elements of them may be one."""
    for d in range(t.dim() - 1):
        if t.shape[d] > 1 and t.stride(d) < t.shape[-1]:
            raise ValueError(f"{name}: elements of an output may not share memory")


# ---------------------------------------------------------------- recurrence
def linear_recurrence(a, x, h0=None, lengths=None, *, gate=True, reverse=False, save=False, out=None, state=None):
    """h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(a), or (``gate`` false) h_t = a_t h_{t-1} + x_t.

    a, x: [T, B, D]; h0: fp32 [B, D] or None (zeros); lengths: int32 [B] on the device or None; ``reverse``: every sequence from its
    last step to its first.  Returns (h, hT, states): h [T, B, D] (zero behind a sequence's end), hT fp32 [B, D] the state behind
    the last step, states fp32 [ceil(T / 16), B, D] for the backward pass with ``save``, else None.  ``out``: a tensor for h;
    ``state``: a contiguous one for hT, which may be h0 itself (a step of generation updates its state in place)."""
    dev = _device(a)
    T, B, D = a.shape
    dt = _type(a, "a")
    pa, px = _want(a, "a", a.shape, a.dtype, dev), _want(x, "x", a.shape, a.dtype, dev)
    p0 = _want(h0, "h0", (B, D), torch.float32, dev, True, True)
    pl = _want(lengths, "lengths", (B,), torch.int32, dev, True, True)
    if out is None:
        out = torch.empty((T, B, D), dtype=a.dtype, device=dev)
    else:
        _own_steps(out, "out")
    if state is None:
        state = torch.empty((B, D), dtype=torch.float32, device=dev)
    states = torch.empty((-(-T // LSTM_LINREC_SEGMENT), B, D), dtype=torch.float32, device=dev) if save else None
    flags = (LSTM_LINREC_GATE if gate else 0) | (LSTM_LINREC_REVERSE if reverse else 0)
    with _On(dev) as stream:
        _check(_b.lstm_linear_recurrence(pa, a.stride(0), a.stride(1), px, x.stride(0), x.stride(1), p0, pl, T, B, D, dt, flags,
                                         _want(out, "out", a.shape, a.dtype, dev), out.stride(0), out.stride(1),
                                         _want(state, "state", (B, D), torch.float32, dev, True), 0 if states is None else states.data_ptr(),
                                         stream))
    return out, state, states


def linear_recurrence_backward(a, x, states, dh, dhT=None, lengths=None, *, gate=True, reverse=False):
    """Gradients of linear_recurrence from its inputs, the ``states`` that it saved, dh [T, B, D] and dhT fp32 [B, D] (or None):
    (da, dx, dh0), da and dx like a, dh0 fp32 [B, D]."""
    dev = _device(a)
    T, B, D = a.shape
    dt = _type(a, "a")
    pa, px, pd = (_want(t, n, a.shape, a.dtype, dev) for t, n in ((a, "a"), (x, "x"), (dh, "dh")))
    ps = _want(states, "states", (-(-T // LSTM_LINREC_SEGMENT), B, D), torch.float32, dev, True)
    pT = _want(dhT, "dhT", (B, D), torch.float32, dev, True, True)
    pl = _want(lengths, "lengths", (B,), torch.int32, dev, True, True)
    da, dx = (torch.empty((T, B, D), dtype=a.dtype, device=dev) for _ in range(2))
    dh0 = torch.empty((B, D), dtype=torch.float32, device=dev)
    flags = (LSTM_LINREC_GATE if gate else 0) | (LSTM_LINREC_REVERSE if reverse else 0)
    with _On(dev) as stream:
        _check(_b.lstm_linear_recurrence_backward(pa, a.stride(0), a.stride(1), px, x.stride(0), x.stride(1), ps, pd, dh.stride(0), dh.stride(1),
                                                  pT, pl, T, B, D, dt, flags, da.data_ptr(), B * D, D, dx.data_ptr(), B * D, D, dh0.data_ptr(),
                                                  stream))
    return da, dx, dh0


# ---------------------------------------------------------------- norm
def _rows(x, w, name):
    dev = _device(x)
    rows, width = x.shape
    return dev, rows, width, _type(x, name), _want(x, name, x.shape, x.dtype, dev), _want(w, "weight", (width,), torch.float32, dev, True)


def rms_norm(x, weight, residual=None, *, eps=1e-6):
    """r = x + residual (x without one), y = r / sqrt(mean(r^2) + eps) * weight over the rows of x [rows, width].
    Returns (y, r), both of x's type; r is None without a residual."""
    dev, rows, width, dt, px, pw = _rows(x, weight, "x")
    y = torch.empty((rows, width), dtype=x.dtype, device=dev)
    r = None if residual is None else torch.empty_like(y)
    pr = _want(residual, "residual", x.shape, x.dtype, dev, optional=True)
    with _On(dev) as stream:
        _check(_b.lstm_rms_norm(px, x.stride(0), pr, residual.stride(0) if pr else 0, pw, eps, rows, width, dt, y.data_ptr(), width, 0,
                                0 if r is None else r.data_ptr(), width, stream))
    return y, r


def _new_bytes(rows, width, dev):
    """Rows of 8-bit values that start on 16 bytes."""
    return torch.empty((rows, (width + 15) // 16 * 16), dtype=torch.float8_e4m3fn, device=dev)


def rms_norm_fp8(x, weight, residual=None, *, eps=1e-6):
    """rms_norm whose y is held in 8 bits, as fp8_product takes it: (q, scales, r), q float8_e4m3fn [rows, width] with rows a multiple
    of 16 bytes apart, scales fp32 [rows, ceil(width / 128)]."""
    dev, rows, width, dt, px, pw = _rows(x, weight, "x")
    held = _new_bytes(rows, width, dev)
    scales = torch.empty((rows, (width + 127) // 128), dtype=torch.float32, device=dev)
    r = None if residual is None else torch.empty((rows, width), dtype=x.dtype, device=dev)
    pr = _want(residual, "residual", x.shape, x.dtype, dev, optional=True)
    with _On(dev) as stream:
        _check(_b.lstm_rms_norm(px, x.stride(0), pr, residual.stride(0) if pr else 0, pw, eps, rows, width, dt, held.data_ptr(), held.stride(0),
                                scales.data_ptr(), 0 if r is None else r.data_ptr(), width, stream))
    return held[:, :width], scales, r


def rms_norm_backward(dy, r, weight, dr=None, *, eps=1e-6):
    """Gradients of rms_norm at r (x where there was no residual): dy and dr (what reaches r past the norm, or None) like r.
    Returns (dx, dw): dx, of x and of the residual alike, of r's type, dw fp32 [width]."""
    dev, rows, width, dt, pr, pw = _rows(r, weight, "r")
    py, pd = _want(dy, "dy", r.shape, r.dtype, dev), _want(dr, "dr", r.shape, r.dtype, dev, optional=True)
    dx = torch.empty((rows, width), dtype=r.dtype, device=dev)
    dw = torch.empty((width,), dtype=torch.float32, device=dev)
    with _On(dev) as stream:
        need = max(_b.lstm_rms_norm_workspace(rows, width), 0)
        workspace = torch.empty((need,), dtype=torch.float32, device=dev)
        _check(_b.lstm_rms_norm_backward(py, dy.stride(0), pr, r.stride(0), pw, pd, dr.stride(0) if pd else 0, eps, rows, width, dt,
                                         dx.data_ptr(), width, dw.data_ptr(), workspace.data_ptr(), need, stream))
    return dx, dw


# ---------------------------------------------------------------- 8-bit matrices
def fp8_quantize(x, *, block_rows=1):
    """x [rows, width] as (q, scales) with x ~ scale * q: a scale for each 128 columns of a row (``block_rows`` 1: activations,
    scales [rows, ceil(width / 128)]) or for each 128 x 128 block (128: weights, scales [ceil(rows / 128), ceil(width / 128)])."""
    dev = _device(x)
    rows, width = x.shape
    dt = _type(x, "x")
    px = _want(x, "x", x.shape, x.dtype, dev)
    held = _new_bytes(rows, width, dev)
    scales = torch.empty(((rows + block_rows - 1) // block_rows if block_rows > 0 else 0, (width + 127) // 128), dtype=torch.float32, device=dev)
    with _On(dev) as stream:
        _check(_b.lstm_fp8_quantize(px, x.stride(0), rows, width, dt, block_rows, held.data_ptr(), held.stride(0), scales.data_ptr(), stream))
    return held[:, :width], scales


def fp8_product(qx, sx, qw, sw, bias=None, *, dtype=torch.bfloat16, out=None):
    """y = x w^T + bias of 8-bit matrices: qx [rows, width] with sx (block_rows 1), qw [outs, width] with sw (block_rows 128), bias
    fp32 [outs] or None; y [rows, outs] of ``dtype``.  Rows of qx and qw are a multiple of 16 bytes apart, as fp8_quantize and
    rms_norm_fp8 make them."""
    dev = _device(qx)
    rows, width = qx.shape
    outs = qw.shape[0]
    blocks = (width + 127) // 128
    f8 = torch.float8_e4m3fn
    px, pw = _want(qx, "qx", qx.shape, f8, dev), _want(qw, "qw", (outs, width), f8, dev)
    psx = _want(sx, "sx", (rows, blocks), torch.float32, dev, True)
    psw = _want(sw, "sw", ((outs + 127) // 128, blocks), torch.float32, dev, True)
    pb = _want(bias, "bias", (outs,), torch.float32, dev, True, True)
    if out is None:
        out = torch.empty((rows, outs), dtype=dtype, device=dev)
    else:
        _own_steps(out, "out")
    py = _want(out, "out", (rows, outs), dtype, dev)
    with _On(dev) as stream:
        _check(_b.lstm_fp8_product(px, _ld(qx), psx, pw, _ld(qw), psw, pb, rows, outs, width, _type(out, "out"), py, out.stride(0), stream))
    return out


def _ld(q):
    """Row stride of 8-bit rows; a single row has any."""
    return q.stride(0) if q.shape[0] > 1 else (q.shape[1] + 15) // 16 * 16
