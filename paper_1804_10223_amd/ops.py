"""Operators of a layer around a recurrence, on sequences [T, B, H]: selective scan, causal convolution, norm, 8-bit projection.

The names mirror the second half of ``include/sprnn.h``; like ``binding`` this module only checks and marshals arguments,
and every call enqueues HIP kernels on torch's current stream of the tensors' device.  Activations are float32, float16
or bfloat16 CUDA tensors whose last dimension is contiguous (the first two may have any strides: batch-major tensors and a
range of the channels of a wider tensor need no copy); parameters and states are contiguous float32 tensors.  Outputs
that the caller does not pass are allocated here, contiguous.  ``lengths`` (int32 [B], on the device) ends samples early:
inputs behind a sample's end are not used, outputs there are zero.  Nothing here takes part in autograd: the backward
passes are calls of their own, like those of ``SparseRNN``.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from .binding import SPRNN_OK, SprnnError, load_library

TYPES = {"float32": 0, "float16": 1, "bfloat16": 2, "float8_e4m3fn": 3}


class Seq(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("step", ctypes.c_int64), ("sample", ctypes.c_int64)]


class Scan(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("channels", ctypes.c_int), ("states", ctypes.c_int),
                ("groups", ctypes.c_int), ("type", ctypes.c_int), ("softplus", ctypes.c_int),
                ("u", Seq), ("dt", Seq), ("z", Seq), ("B", Seq), ("C", Seq),
                ("A", ctypes.c_void_p), ("D", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p), ("lengths", ctypes.c_void_p)]


class ScanGradientBuffers(ctypes.Structure):
    _fields_ = [("u", Seq), ("dt", Seq), ("z", Seq), ("B", Seq), ("C", Seq),
                ("A", ctypes.c_void_p), ("D", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p), ("state", ctypes.c_void_p)]


class Conv(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("channels", ctypes.c_int), ("width", ctypes.c_int),
                ("type", ctypes.c_int), ("silu", ctypes.c_int), ("x", Seq),
                ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("state", ctypes.c_void_p), ("lengths", ctypes.c_void_p)]


class Norm(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("width", ctypes.c_int), ("type", ctypes.c_int),
                ("residual_type", ctypes.c_int), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p)]


class Product(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("rows", ctypes.c_int), ("inputs", ctypes.c_int),
                ("x", Seq), ("x_scales", ctypes.c_void_p), ("w", ctypes.c_void_p), ("w_scales", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


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
        P = ctypes.POINTER
        for name, args in (("sprnn_scan_sizes", [P(Scan), i64p, i64p, i64p]),
                           ("sprnn_scan_forward", [ci, P(Scan), vp, Seq, vp, vp, vp, i64, vp]),
                           ("sprnn_scan_backward", [ci, P(Scan), Seq, vp, vp, P(ScanGradientBuffers), vp, i64, vp]),
                           ("sprnn_conv_forward", [ci, P(Conv), Seq, vp, vp]),
                           ("sprnn_conv_sizes", [P(Conv), i64p]),
                           ("sprnn_conv_backward", [ci, P(Conv), Seq, vp, Seq, vp, vp, vp, vp, i64, vp]),
                           ("sprnn_rms_norm", [ci, P(Norm), Seq, Seq, Seq, ci, Seq, vp, vp]),
                           ("sprnn_rms_norm_sizes", [P(Norm), i64p]),
                           ("sprnn_rms_norm_backward", [ci, P(Norm), Seq, Seq, Seq, Seq, vp, vp, i64, vp]),
                           ("sprnn_project_quantized", [ci, P(Product), ci, Seq, vp])):
            function = getattr(lib, name)
            function.restype, function.argtypes = ci, args
        _lib = lib
    return _lib


def _check(rc, what):
    if rc != SPRNN_OK:
        raise SprnnError(rc, what)


def _type(dtype, what, also=()):
    name = str(dtype).replace("torch.", "")
    if name not in ("float32", "float16", "bfloat16") and name not in also:
        raise TypeError("%s must be float32, float16 or bfloat16%s, got %s" % (what, "".join(", " + a for a in also), name))
    return TYPES[name]


class _Call:
    """The device, stream and shape checks that the arguments of one call share."""

    def __init__(self, first, what):
        import torch
        self.torch = torch
        if not (isinstance(first, torch.Tensor) and first.is_cuda):
            raise TypeError("%s must be a CUDA tensor" % what)
        self.device = first.device
        self.index = first.device.index

    def stream(self):
        return ctypes.c_void_p(self.torch.cuda.current_stream(self.device).cuda_stream)

    def empty(self, shape, dtype):
        return self.torch.empty(shape, dtype=dtype, device=self.device)

    def workspace(self, size):
        """A buffer of this call alone: torch's allocator hands it on in stream order, and a captured graph has its own."""
        return self.empty((max(int(size), 1),), self.torch.uint8)

    def _tensor(self, t, shape, dtype, what):
        if not (isinstance(t, self.torch.Tensor) and t.device == self.device and t.dtype == dtype):
            raise TypeError("%s must be a %s tensor on %s" % (what, str(dtype).replace("torch.", ""), self.device))
        if tuple(t.shape) != tuple(shape):
            raise ValueError("%s must have shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))

    def plain(self, t, shape, dtype, what):
        """Address of a contiguous tensor, or None."""
        if t is None:
            return None
        self._tensor(t, shape, dtype, what)
        if not t.is_contiguous():
            raise TypeError("%s must be contiguous" % what)
        return ctypes.c_void_p(t.data_ptr())

    def seq(self, t, shape, dtype, what):
        """View of a tensor [T, B, ...] whose dimensions behind the second are contiguous, or of none."""
        if t is None:
            return Seq(None, 0, 0)
        self._tensor(t, shape, dtype, what)
        inner = 1
        for d in range(len(shape) - 1, 1, -1):
            if shape[d] > 1 and t.stride(d) != inner:
                raise TypeError("%s must be contiguous behind its first two dimensions" % what)
            inner *= shape[d]
        return Seq(t.data_ptr(), t.stride(0), t.stride(1))

    def lengths(self, t, batch):
        return self.plain(t, (batch,), self.torch.int32, "lengths")


# ------------------------------------------------------------------------------------------------------- selective scan

def _scan(call, u, dt, A, B, C, D, z, dt_bias, softplus, lengths):
    f32 = call.torch.float32
    if u.dim() != 3 or B.dim() != 4:
        raise ValueError("u must be [T, B, C] and B must be [T, B, groups, N]")
    T, batch, channels = u.shape
    groups, states = B.shape[2], B.shape[3]
    s = Scan(T, batch, channels, states, groups, _type(u.dtype, "u"), 1 if softplus else 0)
    wide, low = (T, batch, channels), (T, batch, groups, states)
    s.u, s.dt, s.z = call.seq(u, wide, u.dtype, "u"), call.seq(dt, wide, u.dtype, "dt"), call.seq(z, wide, u.dtype, "z")
    s.B, s.C = call.seq(B, low, u.dtype, "B"), call.seq(C, low, u.dtype, "C")
    if A is None:
        raise TypeError("A must be a float32 tensor on %s" % call.device)
    s.A = call.plain(A, (channels, states), f32, "A")
    s.D, s.dt_bias = call.plain(D, (channels,), f32, "D"), call.plain(dt_bias, (channels,), f32, "dt_bias")
    s.lengths = call.lengths(lengths, batch)
    return s


def scan_sizes(steps, batch, channels, states, groups=1):
    """sprnn_scan_sizes: bytes of (forward workspace, backward workspace, what the forward pass keeps)."""
    s = Scan(steps, batch, channels, states, groups)
    sizes = [ctypes.c_int64() for _ in range(3)]
    _check(_library().sprnn_scan_sizes(ctypes.byref(s), *[ctypes.byref(x) for x in sizes]), "sprnn_scan_sizes")
    return tuple(x.value for x in sizes)


def selective_scan(u, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, state=None, lengths=None, keep=False,
                   out=None, state_out=None):
    """sprnn_scan_forward: u, dt, z [T, B, C], A [C, N], B, C [T, B, groups, N], D, dt_bias [C], state [B, C, N]
    -> (y [T, B, C], state behind the last step [B, C, N]), with keep=True also what selective_scan_backward reads.
    state_out may be state itself (the next token of running sequences: T = 1 with the state in place)."""
    call = _Call(u, "u")
    s = _scan(call, u, dt, A, B, C, D, z, dt_bias, softplus, lengths)
    f32, full = call.torch.float32, (s.batch, s.channels, s.states)
    if out is None:
        out = call.empty((s.steps, s.batch, s.channels), u.dtype)
    if state_out is None:
        state_out = call.empty(full, f32)
    need, _, kept_bytes = scan_sizes(s.steps, s.batch, s.channels, s.states, s.groups)
    workspace = call.workspace(need)
    kept = call.workspace(kept_bytes) if keep else None
    rc = _library().sprnn_scan_forward(call.index, ctypes.byref(s), call.plain(state, full, f32, "state"),
                                       call.seq(out, (s.steps, s.batch, s.channels), u.dtype, "out"),
                                       call.plain(state_out, full, f32, "state_out"), kept.data_ptr() if keep else None,
                                       workspace.data_ptr(), workspace.numel(), call.stream())
    _check(rc, "sprnn_scan_forward")
    return (out, state_out, kept) if keep else (out, state_out)


def selective_scan_backward(dy, u, dt, A, B, C, kept, D=None, z=None, dt_bias=None, softplus=True, lengths=None, d_state=None):
    """sprnn_scan_backward: gradients of selective_scan(..., keep=True) for dy [T, B, C] and d_state [B, C, N] (gradient of
    the state behind the last step) -> ScanGradients."""
    call = _Call(u, "u")
    s = _scan(call, u, dt, A, B, C, D, z, dt_bias, softplus, lengths)
    f32, wide, low, full = call.torch.float32, (s.steps, s.batch, s.channels), (s.steps, s.batch, s.groups, s.states), (s.batch, s.channels, s.states)
    _, need, kept_bytes = scan_sizes(s.steps, s.batch, s.channels, s.states, s.groups)
    kept_at = call.plain(kept, (max(kept_bytes, 1),), call.torch.uint8, "kept")
    if kept_at is None:
        raise TypeError("kept must be what selective_scan(..., keep=True) returned")
    g = ScanGradients(call.empty(wide, u.dtype), call.empty(wide, u.dtype), call.empty((s.channels, s.states), f32),
                      call.empty(low, u.dtype), call.empty(low, u.dtype), None if D is None else call.empty((s.channels,), f32),
                      None if z is None else call.empty(wide, u.dtype), None if dt_bias is None else call.empty((s.channels,), f32),
                      call.empty(full, f32))
    at = lambda t: None if t is None else t.data_ptr()
    b = ScanGradientBuffers(call.seq(g.du, wide, u.dtype, "du"), call.seq(g.ddt, wide, u.dtype, "ddt"), call.seq(g.dz, wide, u.dtype, "dz"),
                            call.seq(g.dB, low, u.dtype, "dB"), call.seq(g.dC, low, u.dtype, "dC"),
                            at(g.dA), at(g.dD), at(g.ddt_bias), at(g.dstate))
    workspace = call.workspace(need)
    rc = _library().sprnn_scan_backward(call.index, ctypes.byref(s), call.seq(dy, wide, u.dtype, "dy"),
                                        call.plain(d_state, full, f32, "d_state"), kept_at, ctypes.byref(b),
                                        workspace.data_ptr(), workspace.numel(), call.stream())
    _check(rc, "sprnn_scan_backward")
    return g


# ---------------------------------------------------------------------------------------------------- causal convolution

def _conv(call, x, weight, bias, silu, state, lengths):
    f32 = call.torch.float32
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x must be [T, B, C] and weight must be [C, K]")
    T, batch, channels = x.shape
    width = weight.shape[1]
    c = Conv(T, batch, channels, width, _type(x.dtype, "x"), 1 if silu else 0)
    c.x = call.seq(x, (T, batch, channels), x.dtype, "x")
    c.weight, c.bias = call.plain(weight, (channels, width), f32, "weight"), call.plain(bias, (channels,), f32, "bias")
    c.state = call.plain(state, (max(width - 1, 0), batch, channels), x.dtype, "state")
    c.lengths = call.lengths(lengths, batch)
    return c


def causal_conv(x, weight, bias=None, silu=True, state=None, lengths=None, out=None, state_out=None):
    """sprnn_conv_forward: x [T, B, C], weight [C, K] (K 1..8), bias [C], state [K - 1, B, C] (the inputs before step 0)
    -> (y [T, B, C], the last K - 1 inputs [K - 1, B, C]).  state_out may be state itself."""
    call = _Call(x, "x")
    c = _conv(call, x, weight, bias, silu, state, lengths)
    wide, past = (c.steps, c.batch, c.channels), (max(c.width - 1, 0), c.batch, c.channels)
    if out is None:
        out = call.empty(wide, x.dtype)
    if state_out is None:
        state_out = call.empty(past, x.dtype)
    rc = _library().sprnn_conv_forward(call.index, ctypes.byref(c), call.seq(out, wide, x.dtype, "out"),
                                       call.plain(state_out, past, x.dtype, "state_out"), call.stream())
    _check(rc, "sprnn_conv_forward")
    return out, state_out


def causal_conv_backward(dy, x, weight, bias=None, silu=True, state=None, lengths=None, d_state=None):
    """sprnn_conv_backward: (dx [T, B, C], dweight [C, K], dbias [C] or None, dstate [K - 1, B, C]) of causal_conv for dy
    [T, B, C] and d_state [K - 1, B, C], the gradient of the state it returned."""
    call = _Call(x, "x")
    c = _conv(call, x, weight, bias, silu, state, lengths)
    f32, wide, past = call.torch.float32, (c.steps, c.batch, c.channels), (max(c.width - 1, 0), c.batch, c.channels)
    need = ctypes.c_int64()
    _check(_library().sprnn_conv_sizes(ctypes.byref(c), ctypes.byref(need)), "sprnn_conv_sizes")
    workspace = call.workspace(need.value)
    dx, dweight, dstate = call.empty(wide, x.dtype), call.empty((c.channels, c.width), f32), call.empty(past, x.dtype)
    dbias = None if bias is None else call.empty((c.channels,), f32)
    rc = _library().sprnn_conv_backward(call.index, ctypes.byref(c), call.seq(dy, wide, x.dtype, "dy"),
                                        call.plain(d_state, past, x.dtype, "d_state"), call.seq(dx, wide, x.dtype, "dx"),
                                        dweight.data_ptr(), None if dbias is None else dbias.data_ptr(), dstate.data_ptr(),
                                        workspace.data_ptr(), workspace.numel(), call.stream())
    _check(rc, "sprnn_conv_backward")
    return dx, dweight, dbias, dstate


# ------------------------------------------------------------------------------------------------------------------ norm

def _norm(call, width, batch, steps, dtype, residual_dtype, eps, weight):
    n = Norm(steps, batch, width, _type(dtype, "x"), _type(residual_dtype, "the residual"), float(eps))
    if residual_dtype not in (dtype, call.torch.float32):
        raise TypeError("the residual must have the type of x or float32")
    n.weight = call.plain(weight, (width,), call.torch.float32, "weight")
    return n


def _norm_forward(x, weight, eps, residual, residual_out, y, y_type, scales):
    call = _Call(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be [T, B, W]")
    shape = tuple(x.shape)
    stream = x.dtype if residual is None else residual.dtype
    n = _norm(call, shape[2], shape[1], shape[0], x.dtype, stream, eps, weight)
    if residual_out is None and residual is not None:
        residual_out = call.empty(shape, stream)
    if y is None:
        y = call.empty(shape, call.torch.float8_e4m3fn if y_type == 3 else x.dtype)
    blocks = (shape[0], shape[1], (shape[2] + 127) // 128)
    if y_type == 3 and scales is None:
        scales = call.empty(blocks, call.torch.float32)
    rc = _library().sprnn_rms_norm(call.index, ctypes.byref(n), call.seq(x, shape, x.dtype, "x"), call.seq(residual, shape, stream, "residual"),
                                   call.seq(residual_out, shape, stream, "residual_out"), n.type if y_type is None else y_type,
                                   call.seq(y, shape, call.torch.float8_e4m3fn if y_type == 3 else x.dtype, "out"),
                                   call.plain(scales, blocks, call.torch.float32, "scales") if y_type == 3 else None, call.stream())
    _check(rc, "sprnn_rms_norm")
    return y, scales, residual_out


def rms_norm(x, weight=None, eps=1e-5, residual=None, residual_out=None, out=None):
    """sprnn_rms_norm: x [T, B, W], residual [T, B, W] (the type of x, or float32) -> (y [T, B, W], x + residual), the
    second None without a residual (and without residual_out).  residual_out may be residual itself."""
    y, _, r = _norm_forward(x, weight, eps, residual, residual_out, out, None, None)
    return y, r


def rms_norm_fp8(x, weight=None, eps=1e-5, residual=None, residual_out=None, out=None, scales=None):
    """sprnn_rms_norm with its output in 8 bits: (y float8_e4m3fn [T, B, W], scales float32 [T, B, ceil(W / 128)],
    x + residual or None); y times the scale of its block of 128 is the normed row."""
    return _norm_forward(x, weight, eps, residual, residual_out, out, 3, scales)


def rms_norm_backward(dy, r, weight=None, eps=1e-5, d_residual=None, dr=None):
    """sprnn_rms_norm_backward: dy [T, B, W], the normed rows r [T, B, W] (x + residual, or x), d_residual (gradient of r
    from elsewhere) -> (gradient of r in the type of r, dweight [W] or None)."""
    call = _Call(dy, "dy")
    if dy.dim() != 3:
        raise ValueError("dy must be [T, B, W]")
    shape = tuple(dy.shape)
    if not isinstance(r, call.torch.Tensor):
        raise TypeError("r must be a CUDA tensor")
    n = _norm(call, shape[2], shape[1], shape[0], dy.dtype, r.dtype, eps, weight)
    need = ctypes.c_int64()
    _check(_library().sprnn_rms_norm_sizes(ctypes.byref(n), ctypes.byref(need)), "sprnn_rms_norm_sizes")
    workspace = call.workspace(need.value if weight is not None else 0)
    if dr is None:
        dr = call.empty(shape, r.dtype)
    dweight = None if weight is None else call.empty((shape[2],), call.torch.float32)
    rc = _library().sprnn_rms_norm_backward(call.index, ctypes.byref(n), call.seq(dy, shape, dy.dtype, "dy"), call.seq(r, shape, r.dtype, "r"),
                                            call.seq(d_residual, shape, r.dtype, "d_residual"), call.seq(dr, shape, r.dtype, "dr"),
                                            None if dweight is None else dweight.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                            call.stream())
    _check(rc, "sprnn_rms_norm_backward")
    return dr, dweight


# ------------------------------------------------------------------------------------------------------ 8-bit projection

def project_fp8(x, x_scales, w, w_scales, bias=None, dtype=None, out=None):
    """sprnn_project_quantized: x float8_e4m3fn [T, B, K] with x_scales [T, B, ceil(K / 128)] (as rms_norm_fp8 returns
    them), w float8_e4m3fn [R, K] with w_scales [ceil(R / 128), ceil(K / 128)], bias [R] -> [T, B, R] in dtype (float32
    unless said otherwise: the ``x`` argument of SparseRNN's forward calls)."""
    call = _Call(x, "x")
    f32, e4m3 = call.torch.float32, call.torch.float8_e4m3fn
    if x.dim() != 3 or not isinstance(w, call.torch.Tensor) or w.dim() != 2:
        raise ValueError("x must be [T, B, K] and w must be [R, K]")
    T, batch, inputs = x.shape
    rows = w.shape[0]
    p = Product(T, batch, rows, inputs)
    blocks = (inputs + 127) // 128
    p.x, p.x_scales = call.seq(x, (T, batch, inputs), e4m3, "x"), call.plain(x_scales, (T, batch, blocks), f32, "x_scales")
    p.w, p.w_scales = call.plain(w, (rows, inputs), e4m3, "w"), call.plain(w_scales, ((rows + 127) // 128, blocks), f32, "w_scales")
    p.bias = call.plain(bias, (rows,), f32, "bias")
    if out is None:
        out = call.empty((T, batch, rows), f32 if dtype is None else dtype)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError("out must be a %s tensor" % str(dtype).replace("torch.", ""))
    rc = _library().sprnn_project_quantized(call.index, ctypes.byref(p), _type(out.dtype, "out"), call.seq(out, (T, batch, rows), out.dtype, "out"),
                                            call.stream())
    _check(rc, "sprnn_project_quantized")
    return out
