"""Operators of a layer around a recurrence, on sequences [T, B, H]: selective scan, causal convolution, norm, 8-bit projection.

The names mirror the second half of ``include/sprnn.h``; like ``binding`` this module only checks and marshals arguments,
and every call enqueues HIP kernels on torch's current stream of the tensors' device.  Activations are float32, float16
or bfloat16 CUDA tensors whose last dimension is contiguous (the first two may have any strides: batch-major tensors and a
range of the channels of a wider tensor need no copy); parameters and states are contiguous float32 tensors.  Outputs
that the caller does not pass are allocated here, contiguous; those that are passed must not overlap inputs unless said
otherwise.  ``lengths`` (int32 [B], on the device) ends samples early: inputs behind a sample's end are not used, outputs
there are zero.  Nothing here takes part in autograd: the backward passes are calls of their own, like those of
``SparseRNN``, and a call on tensors that require gradients warns that its results have none (not under ``torch.no_grad``).
"""
from __future__ import annotations

import ctypes
import functools
import struct
import warnings
from typing import NamedTuple, Optional

import torch

from .binding import SPRNN_OK, SprnnError, load_library

TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.float8_e4m3fn: 3}
F32, E4M3 = torch.float32, torch.float8_e4m3fn


class Seq(ctypes.Structure):
    """sprnn_seq_t, passed by value."""
    _fields_ = [("data", ctypes.c_void_p), ("step", ctypes.c_int64), ("sample", ctypes.c_int64)]


# The structures of the C ABI as bytes (a ctypes structure takes five times as long to fill, more than a token's kernels run).
# Addresses are 0 where there is nothing; a view is its address and the strides of its first two dimensions.
_SCAN = struct.Struct("7i4x" + 5 * "Qqq" + "4Q")               # sprnn_scan_t
_SCAN_GRADIENTS = struct.Struct(5 * "Qqq" + "4Q")              # sprnn_scan_gradients_t
_CONV = struct.Struct("6iQqq4Q")                               # sprnn_conv_t
_NORM = struct.Struct("5ifQ")                                  # sprnn_norm_t
_PRODUCT = struct.Struct("4iQqq4Q")                            # sprnn_product_t
_NOTHING = (0, 0, 0)


class ScanGradients(NamedTuple):
    """What selective_scan_backward returns; dD, dz and ddt_bias are None where the scan has no such argument."""
    du: object
    ddt: object
    dA: object
    dB: object
    dC: object
    dD: Optional[object]
    dz: Optional[object]
    ddt_bias: Optional[object]
    dstate: object


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        vp, ci, i64, i64p = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.POINTER(ctypes.c_int64)
        for name, args in (("sprnn_scan_sizes", [vp, i64p, i64p, i64p]),
                           ("sprnn_scan_forward", [ci, vp, vp, Seq, vp, vp, vp, i64, vp]),
                           ("sprnn_scan_backward", [ci, vp, Seq, vp, vp, vp, vp, i64, vp]),
                           ("sprnn_conv_forward", [ci, vp, Seq, vp, vp]),
                           ("sprnn_conv_sizes", [vp, i64p]),
                           ("sprnn_conv_backward", [ci, vp, Seq, vp, Seq, vp, vp, vp, vp, i64, vp]),
                           ("sprnn_rms_norm", [ci, vp, Seq, Seq, Seq, ci, Seq, vp, vp]),
                           ("sprnn_rms_norm_sizes", [vp, i64p]),
                           ("sprnn_rms_norm_backward", [ci, vp, Seq, Seq, Seq, Seq, vp, vp, i64, vp]),
                           ("sprnn_project_quantized", [ci, vp, ci, Seq, vp])):
            function = getattr(lib, name)
            function.restype, function.argtypes = ci, args
        _lib = lib
    return _lib


def _check(rc, what):
    if rc != SPRNN_OK:
        raise SprnnError(rc, what)


def _name(dtype):
    return str(dtype).replace("torch.", "")


def _type(dtype, what):
    code = TYPES.get(dtype, 3)
    if code == 3:
        raise TypeError("%s must be float32, float16 or bfloat16, got %s" % (what, _name(dtype)))
    return code


def _index(t, what):
    """The GPU that a call's first tensor is on."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError("%s must be a CUDA tensor" % what)
    return t.get_device()


def _stream(index):
    """hipStream_t of torch's current stream (without the Stream object that torch.cuda.current_stream makes, 2 us)."""
    return torch._C._cuda_getCurrentRawStream(index)


def _refuse(t, shape, dtype, index, what):
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.get_device() == index):
        raise TypeError("%s must be a %s tensor on cuda:%d" % (what, _name(dtype), index))
    raise ValueError("%s must have shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))


def _plain(t, shape, dtype, index, what):
    """Address of a contiguous tensor, 0 for None."""
    if t is None:
        return 0
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == index):
        _refuse(t, shape, dtype, index, what)
    if not t.is_contiguous():
        raise TypeError("%s must be contiguous" % what)
    return t.data_ptr()


def _seq(t, shape, dtype, index, what):
    """(address, strides of the first two dimensions) of a tensor [T, B, ...] that is contiguous behind them."""
    if t is None:
        return _NOTHING
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == index):
        _refuse(t, shape, dtype, index, what)
    strides = t.stride()
    if len(strides) == 3:
        if strides[2] != 1 and shape[2] != 1:
            raise TypeError("%s must be contiguous behind its first two dimensions" % what)
    elif (strides[3] != 1 and shape[3] != 1) or (strides[2] != shape[3] and shape[2] != 1):
        raise TypeError("%s must be contiguous behind its first two dimensions" % what)
    return t.data_ptr(), strides[0], strides[1]


def _workspace(size, device):
    """A buffer of one call alone: torch's allocator hands it on in stream order, and a captured graph has its own."""
    return torch.empty((size,), dtype=torch.uint8, device=device) if size else None


def _leads(t):
    return getattr(t, "requires_grad", False)         # (what is no tensor is refused by name later)


def _warn(what, level=3):
    warnings.warn("%s: an argument requires gradients, the results have no graph (the gradients are a call of their own; use "
                  "torch.no_grad or detach where none are wanted)" % what, stacklevel=level)


def _at(t):
    return 0 if t is None else t.data_ptr()


@functools.lru_cache(maxsize=256)
def _sizes(function, head, count):
    """Bytes of the buffers of a call of these sizes (they follow from the sizes alone)."""
    sizes = [ctypes.c_int64() for _ in range(count)]
    _check(getattr(_library(), function)(head, *[ctypes.byref(x) for x in sizes]), function)
    return tuple(x.value for x in sizes)


# ------------------------------------------------------------------------------------------------------- selective scan

@functools.lru_cache(maxsize=256)
def scan_sizes(steps, batch, channels, states, groups=1):
    """sprnn_scan_sizes: bytes of (forward workspace, backward workspace, what the forward pass keeps)."""
    return _sizes("sprnn_scan_sizes", _SCAN.pack(steps, batch, channels, states, groups, *([0] * 21)), 3)


def _scan(index, u, dt, A, B, C, D, z, dt_bias, softplus, lengths):
    """sprnn_scan_t and the sizes (T, batch, C, N, groups)."""
    if not isinstance(B, torch.Tensor):
        raise TypeError("B must be a tensor on cuda:%d" % index)
    if u.dim() != 3 or B.dim() != 4:
        raise ValueError("u must be [T, B, C] and B must be [T, B, groups, N]")
    dtype = u.dtype
    wide, low = u.shape, B.shape
    T, batch, channels = wide
    groups, states = low[2], low[3]
    low = (T, batch, groups, states)
    if A is None or dt is None or C is None:
        raise TypeError("dt, A and C must be tensors on cuda:%d" % index)
    packed = _SCAN.pack(T, batch, channels, states, groups, _type(dtype, "u"), 1 if softplus else 0,
                        *_seq(u, wide, dtype, index, "u"), *_seq(dt, wide, dtype, index, "dt"), *_seq(z, wide, dtype, index, "z"),
                        *_seq(B, low, dtype, index, "B"), *_seq(C, low, dtype, index, "C"),
                        _plain(A, (channels, states), F32, index, "A"), _plain(D, (channels,), F32, index, "D"),
                        _plain(dt_bias, (channels,), F32, index, "dt_bias"), _plain(lengths, (batch,), torch.int32, index, "lengths"))
    return packed, T, batch, channels, states, groups


def selective_scan(u, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, state=None, lengths=None, keep=False,
                   out=None, state_out=None):
    """sprnn_scan_forward: u, dt, z [T, B, C], A [C, N], B, C [T, B, groups, N], D, dt_bias [C], state [B, C, N]
    -> (y [T, B, C], state behind the last step [B, C, N]), with keep=True also what selective_scan_backward reads.
    state_out may be state itself (the next token of running sequences: T = 1 with the state in place)."""
    index = _index(u, "u")
    scan, T, batch, channels, states, groups = _scan(index, u, dt, A, B, C, D, z, dt_bias, softplus, lengths)
    if torch.is_grad_enabled() and (
            u.requires_grad or dt.requires_grad or A.requires_grad or B.requires_grad or C.requires_grad or _leads(D) or _leads(z) or
            _leads(dt_bias) or _leads(state)):
        _warn("selective_scan")
    dtype, device, full = u.dtype, u.device, (batch, channels, states)
    if out is None:
        out = torch.empty((T, batch, channels), dtype=dtype, device=device)
    if state_out is None:
        state_out = torch.empty(full, dtype=F32, device=device)
    need, _, kept_bytes = scan_sizes(T, batch, channels, states, groups)
    workspace = _workspace(need, device)
    kept = torch.empty((kept_bytes,), dtype=torch.uint8, device=device) if keep else None
    rc = _library().sprnn_scan_forward(index, scan, _plain(state, full, F32, index, "state"),
                                       Seq(*_seq(out, (T, batch, channels), dtype, index, "out")),
                                       _plain(state_out, full, F32, index, "state_out"), _at(kept), _at(workspace), need, _stream(index))
    _check(rc, "sprnn_scan_forward")
    return (out, state_out, kept) if keep else (out, state_out)


def selective_scan_backward(dy, u, dt, A, B, C, kept, D=None, z=None, dt_bias=None, softplus=True, lengths=None, d_state=None):
    """sprnn_scan_backward: gradients of selective_scan(..., keep=True) for dy [T, B, C] and d_state [B, C, N] (gradient of
    the state behind the last step) -> ScanGradients."""
    index = _index(u, "u")
    scan, T, batch, channels, states, groups = _scan(index, u, dt, A, B, C, D, z, dt_bias, softplus, lengths)
    dtype, device = u.dtype, u.device
    wide, low, full = (T, batch, channels), (T, batch, groups, states), (batch, channels, states)
    _, need, kept_bytes = scan_sizes(T, batch, channels, states, groups)
    if kept is None:
        raise TypeError("kept must be what selective_scan(..., keep=True) returned")
    kept_at = _plain(kept, (kept_bytes,), torch.uint8, index, "kept")
    empty = lambda shape, type: torch.empty(shape, dtype=type, device=device)
    g = ScanGradients(empty(wide, dtype), empty(wide, dtype), empty((channels, states), F32), empty(low, dtype), empty(low, dtype),
                      None if D is None else empty((channels,), F32), None if z is None else empty(wide, dtype),
                      None if dt_bias is None else empty((channels,), F32), empty(full, F32))
    rows = lambda t: _NOTHING if t is None else (t.data_ptr(),) + t.stride()[:2]
    buffers = _SCAN_GRADIENTS.pack(*rows(g.du), *rows(g.ddt), *rows(g.dz), *rows(g.dB), *rows(g.dC), _at(g.dA), _at(g.dD), _at(g.ddt_bias),
                                   _at(g.dstate))
    workspace = _workspace(need, device)
    rc = _library().sprnn_scan_backward(index, scan, Seq(*_seq(dy, wide, dtype, index, "dy")), _plain(d_state, full, F32, index, "d_state"),
                                        kept_at, buffers, _at(workspace), need, _stream(index))
    _check(rc, "sprnn_scan_backward")
    return g


# ---------------------------------------------------------------------------------------------------- causal convolution

def _conv(index, x, weight, bias, silu, state, lengths):
    """sprnn_conv_t and the sizes (T, batch, C, K)."""
    if not isinstance(weight, torch.Tensor):
        raise TypeError("weight must be a tensor on cuda:%d" % index)
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x must be [T, B, C] and weight must be [C, K]")
    T, batch, channels = x.shape
    width = weight.shape[1]
    packed = _CONV.pack(T, batch, channels, width, _type(x.dtype, "x"), 1 if silu else 0, *_seq(x, x.shape, x.dtype, index, "x"),
                        _plain(weight, (channels, width), F32, index, "weight"), _plain(bias, (channels,), F32, index, "bias"),
                        _plain(state, (max(width - 1, 0), batch, channels), x.dtype, index, "state"),
                        _plain(lengths, (batch,), torch.int32, index, "lengths"))
    return packed, T, batch, channels, width


def causal_conv(x, weight, bias=None, silu=True, state=None, lengths=None, out=None, state_out=None):
    """sprnn_conv_forward: x [T, B, C], weight [C, K] (K 1..8), bias [C], state [K - 1, B, C] (the inputs before step 0)
    -> (y [T, B, C], the last K - 1 inputs [K - 1, B, C]).  state_out may be state itself."""
    index = _index(x, "x")
    conv, T, batch, channels, width = _conv(index, x, weight, bias, silu, state, lengths)
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or _leads(bias) or _leads(state)):
        _warn("causal_conv")
    dtype, wide, past = x.dtype, (T, batch, channels), (max(width - 1, 0), batch, channels)
    if out is None:
        out = torch.empty(wide, dtype=dtype, device=x.device)
    if state_out is None:
        state_out = torch.empty(past, dtype=dtype, device=x.device)
    rc = _library().sprnn_conv_forward(index, conv, Seq(*_seq(out, wide, dtype, index, "out")),
                                       _plain(state_out, past, dtype, index, "state_out"), _stream(index))
    _check(rc, "sprnn_conv_forward")
    return out, state_out


def causal_conv_backward(dy, x, weight, bias=None, silu=True, state=None, lengths=None, d_state=None):
    """sprnn_conv_backward: (dx [T, B, C], dweight [C, K], dbias [C] or None, dstate [K - 1, B, C]) of causal_conv for dy
    [T, B, C] and d_state [K - 1, B, C], the gradient of the state it returned."""
    index = _index(x, "x")
    conv, T, batch, channels, width = _conv(index, x, weight, bias, silu, state, lengths)
    dtype, device, wide, past = x.dtype, x.device, (T, batch, channels), (max(width - 1, 0), batch, channels)
    (need,) = _sizes("sprnn_conv_sizes", _CONV.pack(T, batch, channels, width, *([0] * 9)), 1)
    workspace = _workspace(need, device)
    dx, dstate = torch.empty(wide, dtype=dtype, device=device), torch.empty(past, dtype=dtype, device=device)
    dweight = torch.empty((channels, width), dtype=F32, device=device)
    dbias = None if bias is None else torch.empty((channels,), dtype=F32, device=device)
    rc = _library().sprnn_conv_backward(index, conv, Seq(*_seq(dy, wide, dtype, index, "dy")), _plain(d_state, past, dtype, index, "d_state"),
                                        Seq(*_seq(dx, wide, dtype, index, "dx")), dweight.data_ptr(), _at(dbias), dstate.data_ptr(),
                                        _at(workspace), need, _stream(index))
    _check(rc, "sprnn_conv_backward")
    return dx, dweight, dbias, dstate


# ------------------------------------------------------------------------------------------------------------------ norm

def _norm(index, shape, dtype, stream_dtype, eps, weight):
    if stream_dtype is not dtype and stream_dtype is not F32:
        raise TypeError("the residual must have the type of x or float32")
    return _NORM.pack(shape[0], shape[1], shape[2], _type(dtype, "x"), _type(stream_dtype, "the residual"), eps,
                      _plain(weight, (shape[2],), F32, index, "weight"))


def _norm_forward(x, weight, eps, residual, residual_out, y, scales, quantized):
    index = _index(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be [T, B, W]")
    shape, dtype, device = x.shape, x.dtype, x.device
    stream_dtype = dtype if residual is None else getattr(residual, "dtype", None)
    norm = _norm(index, shape, dtype, stream_dtype, eps, weight)
    if torch.is_grad_enabled() and (x.requires_grad or _leads(weight) or _leads(residual)):
        _warn("rms_norm_fp8" if quantized else "rms_norm", 4)
    y_dtype, blocks = E4M3 if quantized else dtype, (shape[0], shape[1], (shape[2] + 127) // 128)
    if residual_out is None and residual is not None:
        residual_out = torch.empty(shape, dtype=stream_dtype, device=device)
    if y is None:
        y = torch.empty(shape, dtype=y_dtype, device=device)
    if quantized and scales is None:
        scales = torch.empty(blocks, dtype=F32, device=device)
    rc = _library().sprnn_rms_norm(index, norm, Seq(*_seq(x, shape, dtype, index, "x")), Seq(*_seq(residual, shape, stream_dtype, index, "residual")),
                                   Seq(*_seq(residual_out, shape, stream_dtype, index, "residual_out")), TYPES[y_dtype],
                                   Seq(*_seq(y, shape, y_dtype, index, "out")), _plain(scales, blocks, F32, index, "scales"), _stream(index))
    _check(rc, "sprnn_rms_norm")
    return y, scales, residual_out


def rms_norm(x, weight=None, eps=1e-5, residual=None, residual_out=None, out=None):
    """sprnn_rms_norm: x [T, B, W], residual [T, B, W] (the type of x, or float32) -> (y [T, B, W], x + residual), the
    second None without a residual (and without residual_out).  residual_out may be residual itself."""
    y, _, r = _norm_forward(x, weight, eps, residual, residual_out, out, None, False)
    return y, r


def rms_norm_fp8(x, weight=None, eps=1e-5, residual=None, residual_out=None, out=None, scales=None):
    """sprnn_rms_norm with its output in 8 bits: (y float8_e4m3fn [T, B, W], scales float32 [T, B, ceil(W / 128)],
    x + residual or None); y times the scale of its block of 128 is the normed row."""
    return _norm_forward(x, weight, eps, residual, residual_out, out, scales, True)


def rms_norm_backward(dy, r, weight=None, eps=1e-5, d_residual=None, dr=None):
    """sprnn_rms_norm_backward: dy [T, B, W], the normed rows r [T, B, W] (x + residual, or x), d_residual (gradient of r
    from elsewhere) -> (gradient of r in the type of r, dweight [W] or None)."""
    index = _index(dy, "dy")
    if dy.dim() != 3:
        raise ValueError("dy must be [T, B, W]")
    if not isinstance(r, torch.Tensor):
        raise TypeError("r must be a CUDA tensor")
    shape, dtype, r_dtype, device = dy.shape, dy.dtype, r.dtype, dy.device
    norm = _norm(index, shape, dtype, r_dtype, eps, weight)
    need = 0 if weight is None else _sizes("sprnn_rms_norm_sizes", _NORM.pack(shape[0], shape[1], shape[2], 0, 0, 0.0, 0), 1)[0]
    workspace = _workspace(need, device)
    if dr is None:
        dr = torch.empty(shape, dtype=r_dtype, device=device)
    dweight = None if weight is None else torch.empty((shape[2],), dtype=F32, device=device)
    rc = _library().sprnn_rms_norm_backward(index, norm, Seq(*_seq(dy, shape, dtype, index, "dy")), Seq(*_seq(r, shape, r_dtype, index, "r")),
                                            Seq(*_seq(d_residual, shape, r_dtype, index, "d_residual")),
                                            Seq(*_seq(dr, shape, r_dtype, index, "dr")), _at(dweight), _at(workspace), need, _stream(index))
    _check(rc, "sprnn_rms_norm_backward")
    return dr, dweight


# ------------------------------------------------------------------------------------------------------ 8-bit projection

def project_fp8(x, x_scales, w, w_scales, bias=None, dtype=None, out=None):
    """sprnn_project_quantized: x float8_e4m3fn [T, B, K] with x_scales [T, B, ceil(K / 128)] (as rms_norm_fp8 returns
    them), w float8_e4m3fn [R, K] with w_scales [ceil(R / 128), ceil(K / 128)], bias [R] -> [T, B, R] in dtype (float32
    unless said otherwise: the ``x`` argument of SparseRNN's forward calls)."""
    index = _index(x, "x")
    if x.dim() != 3 or not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise ValueError("x must be [T, B, K] and w must be [R, K]")
    if x_scales is None or w_scales is None:
        raise TypeError("x_scales and w_scales must be float32 tensors on cuda:%d" % index)
    shape = x.shape
    T, batch, inputs = shape
    rows = w.shape[0]
    blocks = (inputs + 127) // 128
    product = _PRODUCT.pack(T, batch, rows, inputs, *_seq(x, shape, E4M3, index, "x"), _plain(x_scales, (T, batch, blocks), F32, index, "x_scales"),
                            _plain(w, (rows, inputs), E4M3, index, "w"),
                            _plain(w_scales, ((rows + 127) // 128, blocks), F32, index, "w_scales"), _plain(bias, (rows,), F32, index, "bias"))
    if torch.is_grad_enabled() and (x.requires_grad or x_scales.requires_grad or w.requires_grad or w_scales.requires_grad or _leads(bias)):
        _warn("project_fp8")
    if out is None:
        out = torch.empty((T, batch, rows), dtype=F32 if dtype is None else dtype, device=x.device)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError("out must be a %s tensor" % _name(dtype))
    rc = _library().sprnn_project_quantized(index, product, _type(out.dtype, "out"),
                                            Seq(*_seq(out, (T, batch, rows), out.dtype, index, "out")), _stream(index))
    _check(rc, "sprnn_project_quantized")
    return out
