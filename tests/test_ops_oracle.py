"""CPU: the 64-bit definitions that the GPU tests of ops compare with, against autograd and against differences; refusals of
the C entry points and of the Python ones (nothing here reaches a GPU)."""
import ctypes

import pytest
import torch

import ops_oracle as ref
import ops_structures as st
from paper_1804_10223_amd import binding, ops


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float64)


def _scan_inputs(gen, T, B, C, N, G, gate=True):
    return dict(u=_normal(gen, T, B, C), dt=_normal(gen, T, B, C), A=-torch.rand((C, N), generator=gen, dtype=torch.float64) * 2 - 0.1,
                B=_normal(gen, T, B, G, N), C=_normal(gen, T, B, G, N), D=_normal(gen, C), z=_normal(gen, T, B, C) if gate else None,
                dt_bias=_normal(gen, C), state=_normal(gen, B, C, N))


@pytest.mark.parametrize("lengths", [None, [3, 0, 5]])
@pytest.mark.parametrize("gate,softplus", [(True, True), (False, False)])
def test_scan_gradients_are_those_of_autograd_and_of_differences(lengths, gate, softplus):
    gen = torch.Generator().manual_seed(3)
    T, B, C, N, G = 5, 3, 4, 3, 2
    inputs = _scan_inputs(gen, T, B, C, N, G, gate)
    dy, ds = _normal(gen, T, B, C), _normal(gen, B, C, N)
    got = ref.scan(**inputs, softplus=softplus, lengths=lengths, dy=dy, d_state=ds)

    def loss(**over):
        out = ref.scan(**{**inputs, **over}, softplus=softplus, lengths=lengths)
        return (out["y"] * dy).sum() + (out["state"] * ds).sum()

    names = {"u": "du", "dt": "ddt", "A": "dA", "B": "dB", "C": "dC", "D": "dD", "z": "dz", "dt_bias": "ddt_bias", "state": "dstate"}
    for name, grad in names.items():
        if inputs[name] is None:
            continue
        x = inputs[name].clone().requires_grad_()
        (auto,) = torch.autograd.grad(loss(**{name: x}), [x])
        assert torch.allclose(got[grad], auto, rtol=1e-9, atol=1e-10), name
        way = _normal(gen, *x.shape)
        step = 1e-5
        slope = (loss(**{name: inputs[name] + step * way}) - loss(**{name: inputs[name] - step * way})) / (2 * step)
        assert abs(float(slope - (got[grad] * way).sum())) < 1e-6 * (1.0 + abs(float(slope))), name


@pytest.mark.parametrize("lengths", [None, [0, 1, 6]])
@pytest.mark.parametrize("K,silu", [(1, True), (4, True), (3, False)])
def test_conv_gradients_are_those_of_autograd_and_of_differences(lengths, K, silu):
    gen = torch.Generator().manual_seed(4)
    T, B, C = 6, 3, 5
    inputs = dict(x=_normal(gen, T, B, C), weight=_normal(gen, C, K), bias=_normal(gen, C), state=_normal(gen, K - 1, B, C))
    dy, ds = _normal(gen, T, B, C), _normal(gen, K - 1, B, C)
    got = ref.conv(**inputs, silu=silu, lengths=lengths, dy=dy, d_state=ds)

    def loss(**over):
        out = ref.conv(**{**inputs, **over}, silu=silu, lengths=lengths)
        return (out["y"] * dy).sum() + (out["state"] * ds).sum()

    for name, grad in (("x", "dx"), ("weight", "dweight"), ("bias", "dbias"), ("state", "dstate")):
        if not inputs[name].numel():
            continue
        x = inputs[name].clone().requires_grad_()
        (auto,) = torch.autograd.grad(loss(**{name: x}), [x])
        assert torch.allclose(got[grad], auto, rtol=1e-9, atol=1e-10), name
        way, step = _normal(gen, *x.shape), 1e-5
        slope = (loss(**{name: inputs[name] + step * way}) - loss(**{name: inputs[name] - step * way})) / (2 * step)
        assert abs(float(slope - (got[grad] * way).sum())) < 1e-6 * (1.0 + abs(float(slope))), name


def test_norm_gradients_are_those_of_autograd():
    gen = torch.Generator().manual_seed(5)
    r, w, dy, dr = _normal(gen, 2, 3, 7), _normal(gen, 7), _normal(gen, 2, 3, 7), _normal(gen, 2, 3, 7)
    got = ref.norm_backward(dy, r, w, d_residual=dr)
    r_, w_ = r.clone().requires_grad_(), w.clone().requires_grad_()
    want = torch.autograd.grad((ref.norm(r_, w_) * dy).sum() + (r_ * dr).sum(), (r_, w_))
    assert torch.allclose(got[0], want[0], rtol=1e-10, atol=1e-12) and torch.allclose(got[1], want[1], rtol=1e-10, atol=1e-12)


# ---- refusals.  The addresses are never used: the checks come before the first HIP call.
AT = 1 << 20


def _seq(step=8, sample=8, at=AT):
    return ops.Seq(at, step, sample)


def _own(s):
    return st.Seq(s.data, s.step, s.sample)


def _scan_arguments(**over):
    s = st.Scan(4, 1, 8, 4, 2, 0, 1)
    s.u = s.dt = s.B = s.C = _own(_seq())
    s.A = AT
    for k, v in over.items():
        setattr(s, k, _own(v) if isinstance(v, ops.Seq) else v)
    return s


def test_the_packed_structures_are_those_of_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no gcc here")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = {"scan": (st.Scan, ops._SCAN), "scan_gradients": (st.ScanGradientBuffers, ops._SCAN_GRADIENTS), "conv": (st.Conv, ops._CONV),
             "norm": (st.Norm, ops._NORM), "product": (st.Product, ops._PRODUCT)}
    lines = ['printf("%%zu", sizeof(sprnn_%s_t));' % n + "".join(
        'printf(" %%zu", offsetof(sprnn_%s_t, %s));' % (n, field) for field, _ in names[n][0]._fields_) + 'printf("\\n");' for n in names]
    (tmp_path / "sizes.c").write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"sprnn.h\"\nint main(void) {\n%s\nreturn 0;\n}\n" % "\n".join(lines))
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-I" + os.path.join(root, "include"), str(tmp_path / "sizes.c"), "-o", exe], check=True)
    said = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines()
    for (structure, packed), line in zip(names.values(), said):
        size, *offsets = [int(x) for x in line.split()]
        assert size == packed.size == ctypes.sizeof(structure)
        assert offsets == [getattr(structure, field).offset for field, _ in structure._fields_]
    assert ctypes.sizeof(ops.Seq) == ctypes.sizeof(st.Seq) == 24


@pytest.mark.parametrize("over", [dict(steps=-1), dict(steps=(1 << 22) + 1), dict(batch=-1), dict(batch=65536), dict(channels=0),
                                  dict(channels=(1 << 20) + 8), dict(states=0), dict(states=129), dict(groups=0), dict(groups=3),
                                  dict(type=3), dict(type=-1), dict(softplus=2), dict(A=None), dict(A=AT + 2), dict(D=AT + 1),
                                  dict(dt_bias=AT + 2), dict(lengths=AT + 1), dict(u=_seq(at=None)), dict(dt=_seq(at=AT + 1)),
                                  dict(z=_seq(step=-1)), dict(B=_seq(sample=-8)), dict(C=_seq(step=(1 << 25) + 1))])
def test_scan_refuses(over):
    lib = ops._library()
    s = _scan_arguments(**over)
    assert lib.sprnn_scan_forward(0, ctypes.byref(s), None, _seq(), None, None, None, 0, None) == binding.SPRNN_ERR_INVALID
    g = st.ScanGradientBuffers()
    assert lib.sprnn_scan_backward(0, ctypes.byref(s), _seq(), None, AT, ctypes.byref(g), AT, 1 << 40, None) == binding.SPRNN_ERR_INVALID


def test_scan_refuses_buffers():
    lib, bad = ops._library(), binding.SPRNN_ERR_INVALID
    s = _scan_arguments()
    forward = lambda s=s, device=0, state=None, y=_seq(), out=None, kept=None, work=None, size=0: lib.sprnn_scan_forward(
        device, ctypes.byref(s) if s is not None else None, state, y, out, kept, work, size, None)
    assert forward(s=None) == bad and forward(device=-1) == bad and forward(state=AT + 1) == bad and forward(out=AT + 2) == bad
    assert forward(kept=AT + 8) == bad and forward(y=_seq(at=None)) == bad
    assert forward(y=_seq(step=7)) == bad                                  # rows of the output would overlap
    two = _scan_arguments(batch=2)
    assert forward(s=two, y=_seq(step=12, sample=8)) == bad and forward(s=two, y=_seq(step=8, sample=16)) == bad
    long = _scan_arguments(steps=4096)                                     # divided: needs its workspace
    need = ops.scan_sizes(4096, 1, 8, 4, 2)[0]
    assert need > 0
    assert forward(s=long, work=AT, size=need - 1) == bad and forward(s=long, work=None, size=need) == bad
    assert forward(s=long, work=AT + 8, size=need) == bad
    g = st.ScanGradientBuffers()
    backward = lambda s=s, dy=_seq(), state=None, kept=AT, g=g, work=AT, size=1 << 40: lib.sprnn_scan_backward(
        0, ctypes.byref(s), dy, state, kept, ctypes.byref(g) if g is not None else None, work, size, None)
    assert backward(kept=None) == bad and backward(kept=AT + 4) == bad and backward(dy=_seq(at=None)) == bad and backward(g=None) == bad
    assert backward(work=None) == bad and backward(size=ops.scan_sizes(4, 1, 8, 4, 2)[1] - 1) == bad
    assert backward(g=st.ScanGradientBuffers(z=_own(_seq()))) == bad            # a gate's gradient without a gate
    assert backward(g=st.ScanGradientBuffers(u=_own(_seq(step=4)))) == bad
    with pytest.raises(binding.SprnnError):
        ops.scan_sizes(1, 1, 7, 4, 2)


def _conv_arguments(**over):
    c = st.Conv(4, 1, 8, 4, 0, 1)
    c.x, c.weight = _own(_seq()), AT
    for k, v in over.items():
        setattr(c, k, _own(v) if isinstance(v, ops.Seq) else v)
    return c


@pytest.mark.parametrize("over", [dict(steps=-1), dict(batch=65536), dict(channels=0), dict(channels=(1 << 24) + 1), dict(width=0),
                                  dict(width=9), dict(type=3), dict(silu=2), dict(weight=None), dict(weight=AT + 2), dict(bias=AT + 1),
                                  dict(state=AT + 2), dict(lengths=AT + 1), dict(x=_seq(at=None)), dict(x=_seq(step=-1))])
def test_conv_refuses(over):
    lib, bad = ops._library(), binding.SPRNN_ERR_INVALID
    c = _conv_arguments(**over)
    assert lib.sprnn_conv_forward(0, ctypes.byref(c), _seq(), None, None) == bad
    assert lib.sprnn_conv_backward(0, ctypes.byref(c), _seq(), None, _seq(), AT, AT, None, AT, 1 << 40, None) == bad


def test_conv_refuses_buffers():
    lib, bad = ops._library(), binding.SPRNN_ERR_INVALID
    c = _conv_arguments()
    assert lib.sprnn_conv_forward(0, None, _seq(), None, None) == bad
    assert lib.sprnn_conv_forward(-1, ctypes.byref(c), _seq(), None, None) == bad
    assert lib.sprnn_conv_forward(0, ctypes.byref(c), _seq(step=4), None, None) == bad
    assert lib.sprnn_conv_forward(0, ctypes.byref(c), _seq(), AT + 1, None) == bad
    need = ctypes.c_int64()
    assert lib.sprnn_conv_sizes(ctypes.byref(c), ctypes.byref(need)) == 0 and need.value > 0
    assert lib.sprnn_conv_backward(0, ctypes.byref(c), _seq(), None, _seq(), AT, None, None, AT, need.value - 1, None) == bad
    assert lib.sprnn_conv_backward(0, ctypes.byref(c), _seq(), None, _seq(), AT, None, None, None, need.value, None) == bad
    assert lib.sprnn_conv_backward(0, ctypes.byref(c), _seq(at=None), None, _seq(), None, None, None, None, 0, None) == bad
    assert lib.sprnn_conv_backward(0, ctypes.byref(c), _seq(), None, _seq(step=7), None, None, None, None, 0, None) == bad


@pytest.mark.parametrize("over", [dict(steps=-1), dict(batch=-1), dict(width=0), dict(type=3), dict(residual_type=2), dict(eps=-1.0),
                                  dict(eps=float("nan")), dict(weight=AT + 2)])
def test_norm_refuses(over):
    lib, bad = ops._library(), binding.SPRNN_ERR_INVALID
    n = st.Norm(4, 1, 8, 1, 0, 1e-5)
    for k, v in over.items():
        setattr(n, k, v)
    none = ops.Seq()
    assert lib.sprnn_rms_norm(0, ctypes.byref(n), _seq(), none, none, n.type, _seq(), None, None) == bad
    assert lib.sprnn_rms_norm_backward(0, ctypes.byref(n), _seq(), _seq(), none, _seq(), AT, AT, 1 << 40, None) == bad


def test_norm_refuses_buffers():
    lib, bad, none = ops._library(), binding.SPRNN_ERR_INVALID, ops.Seq()
    n = st.Norm(4, 1, 8, 1, 0, 1e-5)
    call = lambda x=_seq(), r=none, ro=none, t=1, y=_seq(), s=None: lib.sprnn_rms_norm(0, ctypes.byref(n), x, r, ro, t, y, s, None)
    assert call(x=none) == bad and call(y=none) == bad and call(t=0) == bad and call(t=2) == bad      # y in another type
    assert call(t=3) == bad and call(t=1, s=AT) == bad and call(t=3, s=AT + 2) == bad                 # scales with e4m3, and only then
    assert call(ro=_seq(step=4)) == bad and call(r=_seq(at=AT + 2)) == bad and call(y=_seq(step=4)) == bad
    need = ctypes.c_int64()
    assert lib.sprnn_rms_norm_sizes(ctypes.byref(n), ctypes.byref(need)) == 0
    back = lambda dy=_seq(), r=_seq(), dr=_seq(), w=AT, work=AT, size=1 << 40: lib.sprnn_rms_norm_backward(
        0, ctypes.byref(n), dy, r, none, dr, w, work, size, None)
    assert back(dy=none) == bad and back(r=none) == bad and back(dr=none) == bad and back(dr=_seq(step=4)) == bad
    assert back(work=None) == bad and back(size=need.value - 1) == bad and back(w=AT + 2) == bad


def test_project_refuses():
    lib, bad = ops._library(), binding.SPRNN_ERR_INVALID

    def call(out_type=0, out=_seq(), **over):
        p = st.Product(4, 1, 8, 16)
        p.x, p.x_scales, p.w, p.w_scales = _own(_seq(16, 16)), AT, AT, AT
        for k, v in over.items():
            setattr(p, k, v)
        return lib.sprnn_project_quantized(0, ctypes.byref(p), out_type, out, None)

    for over in (dict(steps=-1), dict(batch=70000), dict(rows=0), dict(inputs=0), dict(inputs=(1 << 24) + 1), dict(x=st.Seq()),
                 dict(x_scales=None), dict(x_scales=AT + 2), dict(w=None), dict(w_scales=None), dict(w_scales=AT + 1), dict(bias=AT + 2)):
        assert call(**over) == bad, over
    assert call(out_type=3) == bad and call(out=_seq(step=7)) == bad and call(out=ops.Seq()) == bad
    assert lib.sprnn_project_quantized(0, None, 0, _seq(), None) == bad


def test_calls_without_work_succeed_without_a_gpu():
    lib, none = ops._library(), ops.Seq()
    s = _scan_arguments(batch=0, u=_own(none), dt=_own(none), B=_own(none), C=_own(none))
    assert lib.sprnn_scan_forward(0, ctypes.byref(s), None, none, None, None, None, 0, None) == 0
    c = _conv_arguments(batch=0, x=none)
    assert lib.sprnn_conv_forward(0, ctypes.byref(c), none, None, None) == 0
    n = st.Norm(0, 3, 8, 0, 0, 1e-5)
    assert lib.sprnn_rms_norm(0, ctypes.byref(n), none, none, none, 0, none, None, None) == 0
    p = st.Product(0, 3, 8, 16)
    assert lib.sprnn_project_quantized(0, ctypes.byref(p), 0, none, None) == 0


def test_python_entry_points_refuse_what_is_not_on_a_gpu():
    x = torch.zeros((2, 1, 8))
    for call in (lambda: ops.selective_scan(x, x, None, None, None), lambda: ops.causal_conv(x, x[0, 0][:, None]), lambda: ops.rms_norm(x),
                 lambda: ops.rms_norm_backward(x, x), lambda: ops.rms_norm_fp8(None), lambda: ops.project_fp8(x, x, x, x)):
        with pytest.raises(TypeError):
            call()
