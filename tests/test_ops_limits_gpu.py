"""GPU tests of the operators in paper_1804_10223_amd.ops at the ends of what their header allows: values, strides, sizes.

Tolerances are counted as in test_ops_gpu: roundings on the longest path, times half a step of binary32, times the same sums
over absolute values, plus the rounding of the result to its type.
"""
import pytest
import torch

import ops_oracle as ref
import ops_slow_decay as slow
from test_ops_gpu import BF16, F16, F32, TYPES, _close, _double, _ops, _place, _scan_case, _scan_roundings

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------ 8-bit projection

@pytest.mark.parametrize("type", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,B,K,R", [(1, 3, 128, 40), (1, 30, 272, 4500), (1, 64, 200, 100), (20, 10, 256, 5000), (500, 8, 128, 600), (90, 3, 72, 3900)])
def test_projection_sums_that_cancel(T, B, K, R, type):
    """Of eight neighbouring products two are large and cancel, six are 2^-15 of them: their sum is what is left.  Every type
    of output has it, since the sums are binary32 for all of them."""
    ops = _ops()
    gen = torch.Generator().manual_seed(K)
    place = torch.arange(K) % 8
    x = torch.where(place < 2, 256.0, 2.0).repeat(T * B, 1)
    x[:, place == 1] = -256.0
    flip = torch.randint(0, 2, (T * B, 1), generator=gen) * 2.0 - 1.0
    w = torch.where(place < 2, 448.0, 2.0).repeat(R, 1)
    q, wq = (x * flip).to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn)
    blocks = -(-K // 128)
    xs, ws = torch.full((T * B, blocks), 2.0 ** -4), torch.full((-(-R // 128), blocks), 2.0 ** -3)
    want, size = ref.project(q, xs, wq, ws), ref.project(q, xs, wq, ws, absolute=True)
    assert (want.abs() > 20.0 / 128.0 * K / 8.0).all()
    out = ops.project_fp8(q.view(T, B, K).cuda(), xs.view(T, B, blocks).cuda(), wq.cuda(), ws.cuda(), dtype=TYPES[type])
    # the sum of a block of 128 exact products, a scale of two, the sum over blocks: 5e-6 of the absolute sums, where what is
    # left is 1e-4 of them
    n = min(K, 128) + 3 + blocks
    _close(out, want.view(T, B, R), size.view(T, B, R), n, "out")


@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("T,B,K,R", [(1, 8, 2304, 1024), (1, 40, 1152, 4300), (20, 10, 640, 5000), (700, 4, 272, 1700)])
def test_projection_sums_are_binary32_for_every_type(T, B, K, R, type):
    ops = _ops()
    gen = torch.Generator().manual_seed(R)
    normal = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)
    q, xs = ref.blocks(normal(T * B, K), 1, 128)
    w, ws = ref.blocks(normal(R, K) / K ** 0.5, 128, 128)
    b = normal(R).float()
    want, size = ref.project(q, xs, w, ws, b), ref.project(q, xs, w, ws, b, absolute=True)
    out = ops.project_fp8(q.view(T, B, K).cuda(), xs.view(T, B, -1).cuda(), w.cuda(), ws.cuda(), b.cuda(), dtype=TYPES[type])
    _close(out, want.view(T, B, R), size.view(T, B, R), min(K, 128) + 3 + -(-K // 128) + 2, "out")


# ---------------------------------------------------------------------------------------------------------------- scan

def _masked_scan(T, B, C, N, dtype, value, seed):
    """A scan whose every third step is masked in half of the channels by dt = value."""
    case = _scan_case(T, B, C, N, 1, dtype, True, True, True, True, True, None, seed)
    masked = torch.zeros((T, B, C), dtype=torch.bool)
    masked[::3, :, ::2] = True
    case["dt"][masked] = value
    return case, masked


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("value", ["-inf", "lowest"])
@pytest.mark.parametrize("T,B,C,N", [(1, 2, 70, 16), (1, 1, 9, 5), (11, 2, 70, 16), (20, 1, 33, 40), (300, 1, 24, 16), (300, 2, 10, 100)])
def test_scan_steps_masked_by_infinity_and_the_lowest_value(T, B, C, N, value, type):
    """d is 0 there: the state stays, the step's input does not count, and dt has no gradient."""
    ops, dtype = _ops(), TYPES[type]
    case, masked = _masked_scan(T, B, C, N, dtype, float("-inf") if value == "-inf" else torch.finfo(dtype).min, seed=T + C)
    gen = torch.Generator().manual_seed(T)
    dy, ds = torch.randn((T, B, C), generator=gen).to(dtype), torch.randn((B, C, N), generator=gen)
    want = ref.scan(**_double(case), dy=dy.double(), d_state=ds.double())
    size = ref.scan(**_double(case), dy=dy.double(), d_state=ds.double(), absolute=True)
    dev = {k: v.cuda() for k, v in case.items()}
    args = [dev[k] for k in ("u", "dt", "A", "B", "C")]
    rest = {k: dev[k] for k in ("D", "z", "dt_bias")}
    n = _scan_roundings(T, N, C, {**case, "dt": case["dt"][~masked]}, True)
    for keep in (False, True):
        y, s, *kept = ops.selective_scan(*args, state=dev["state"], keep=keep, **rest)
        _close(y, want["y"], size["y"], n + 20, "y")
        _close(s, want["state"], size["state"], n, "state")
    g = ops.selective_scan_backward(dy.cuda(), *args, kept[0], d_state=ds.cuda(), **rest)
    for name, more in (("du", 0), ("ddt", 0), ("dz", 0), ("dB", C), ("dC", C), ("dA", T * B), ("dD", T * B), ("ddt_bias", T * B), ("dstate", 0)):
        _close(getattr(g, name), want[name], size[name], 2 * n + 60 + more, name)
    assert (g.ddt.cpu()[masked] == 0).all()


def test_scan_of_masked_steps_alone_leaves_the_state_and_other_ends_of_dt():
    ops = _ops()
    C, N = 48, 16
    gen = torch.Generator().manual_seed(5)
    for T in (1, 9, 400):
        st = torch.randn((1, C, N), generator=gen).cuda()
        u, low = torch.randn((T, 1, C), generator=gen).cuda(), torch.rand((T, 1, 1, N), generator=gen).cuda() + 0.5
        A = -torch.rand((C, N), generator=gen).cuda() - 0.1
        for value in (float("-inf"), torch.finfo(F32).min, -1e38, -3e38):
            y, s = ops.selective_scan(u, torch.full_like(u, value), A, low, low, state=st)
            assert torch.equal(s, st) and torch.isfinite(y).all()
        # the other end: a step without end forgets the state and takes an infinite input; NaN stays NaN, in its own channel
        dt = torch.zeros_like(u)
        dt[T - 1, 0, 3], dt[T - 1, 0, 7] = float("inf"), float("nan")
        y, s = ops.selective_scan(u.abs() + 0.1, dt, A, low, low, state=st)
        assert (y[T - 1, 0, 3] == float("inf")).all() and (s[0, 3] == float("inf")).all()
        assert torch.isnan(y[T - 1, 0, 7]) and torch.isnan(s[0, 7]).all()
        assert int((~torch.isfinite(y)).sum()) == 2 and int((~torch.isfinite(s)).sum()) == 2 * N


def _one_step(x, step):
    """[1, B, ..] on the GPU with any stride between its steps, of which there is one."""
    x = x.cuda()
    return x.as_strided(x.shape, (step,) + x.stride()[1:])


@pytest.mark.parametrize("step", [0, 1, 5, 37, (1 << 25) + 1, 1 << 31, (1 << 33) - 4])
@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,N", [(3, 70, 16), (2, 20, 3), (2, 130, 40)])
def test_scan_of_one_step_with_any_stride_between_steps(B, C, N, type, step):
    """The stride between steps is no part of a sequence of one step: inputs and outputs may have any, through every entry."""
    import ctypes
    import ops_structures as st
    ops, dtype = _ops(), TYPES[type]
    gen = torch.Generator().manual_seed(C)
    case = _scan_case(1, B, C, N, 1, dtype, True, True, True, True, True, None, C)
    dy, ds = torch.randn((1, B, C), generator=gen).to(dtype).cuda(), torch.randn((B, C, N), generator=gen).cuda()
    dev = {k: v.cuda() for k, v in case.items()}
    args, rest = [dev[k] for k in ("u", "dt", "A", "B", "C")], {k: dev[k] for k in ("D", "z", "dt_bias")}
    y, s, kept = ops.selective_scan(*args, state=dev["state"], keep=True, **rest)
    want = ops.selective_scan_backward(dy, *args, kept, d_state=ds, **rest)
    token, _ = ops.selective_scan(*args, state=dev["state"], **rest)
    size = ref.scan(**_double(case), absolute=True)
    # (the token's kernel has the same roundings in another order)
    assert ((token - y).double().cpu().abs() <= (200 * 2.0 ** -24 + 2 * ref.half_step(dtype)) * size["y"] + 2 * ref.smallest(dtype)).all()

    near = {k: _one_step(case[k], step) for k in ("u", "dt", "B", "C", "z")}
    args = [near["u"], near["dt"], dev["A"], near["B"], near["C"]]
    rest = {"D": dev["D"], "z": near["z"], "dt_bias": dev["dt_bias"]}
    for keep in (False, True):
        out = torch.full((1, B, C), 7.0, dtype=dtype, device="cuda").as_strided((1, B, C), (step, C, 1))
        got = ops.selective_scan(*args, state=dev["state"], keep=keep, out=out, **rest)
        assert torch.equal(out, y if keep else token)
        assert torch.equal(got[1], s) or not keep
    again = ops.selective_scan_backward(_one_step(dy, step), *args, got[2], d_state=ds, **rest)
    assert all(torch.equal(a, b) for a, b in zip(again, want))

    # outputs of the caller's own
    at = lambda t: st.Seq(t.data_ptr(), step, t.stride(1))
    scan = st.Scan(1, B, C, N, 1, {F32: 0, BF16: 2}[dtype], 1, at(near["u"]), at(near["dt"]), at(near["z"]), at(near["B"]), at(near["C"]),
                   dev["A"].data_ptr(), dev["D"].data_ptr(), dev["dt_bias"].data_ptr(), None)
    own = {k: torch.full_like(getattr(want, k), 7.0) for k in ("du", "ddt", "dz", "dB", "dC")}
    g = st.ScanGradientBuffers(*[at(own[k]) for k in ("du", "ddt", "dz", "dB", "dC")], None, None, None, None)
    need = ops.scan_sizes(1, B, C, N, 1)[1]
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert ops._library().sprnn_scan_backward(0, ctypes.byref(scan), ops.Seq(dy.data_ptr(), step, C), ds.data_ptr(), kept.data_ptr(),
                                              ctypes.byref(g), work.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for name, got in own.items():
        assert torch.equal(got, getattr(want, name)), name


# ---------------------------------------------------------------------------------------------------------------- conv

@pytest.mark.parametrize("T", [0, 5])
def test_conv_gradients_without_a_sample_are_zeros(T):
    import ctypes
    import ops_structures as st
    ops = _ops()
    C, K = 70, 4
    weight, bias = torch.ones((C, K), device="cuda"), torch.ones(C, device="cuda")
    conv = st.Conv(T, 0, C, K, 0, 1, st.Seq(None, C, C), weight.data_ptr(), bias.data_ptr(), None, None)
    dw, db = torch.full((C, K), 7.0, device="cuda"), torch.full((C,), 7.0, device="cuda")
    assert ops._library().sprnn_conv_backward(0, ctypes.byref(conv), ops.Seq(), None, ops.Seq(), dw.data_ptr(), db.data_ptr(), None, None, 0,
                                              torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert (dw == 0).all() and (db == 0).all()
    x = torch.zeros((T, 0, C), device="cuda")
    dx, dw, db, ds = ops.causal_conv_backward(x, x, weight, bias)
    assert dx.shape == x.shape and ds.shape == (K - 1, 0, C) and (dw == 0).all() and (db == 0).all()


def test_scan_gradients_of_more_sums_than_a_launch_has_lanes():
    """A group for every channel: 2^32 sums of dB and dC.  Each group is a scan of its own, so a few of them make the reference."""
    import ctypes
    import ops_structures as st
    ops = _ops()
    T, B, C, some = 64, 8, 1 << 20, 64
    gen = torch.Generator().manual_seed(1)
    one = {k: torch.randn(C, generator=gen).to(BF16).cuda() for k in ("u", "dt", "B", "C", "dy")}
    A = -torch.rand((C, 1), generator=gen).cuda() - 0.05
    ends = torch.tensor([64, 1, 33, 64, 0, 7, 64, 64], dtype=torch.int32, device="cuda")

    def backward(part):
        n = A[part].shape[0]
        rows = {k: v[part].expand(T, B, n) for k, v in one.items()}            # every step and sample has the same inputs
        low = {k: rows[k].unsqueeze(-1) for k in ("B", "C")}
        _, _, kept = ops.selective_scan(rows["u"], rows["dt"], A[part], low["B"], low["C"], lengths=ends, keep=True)
        at = lambda t: st.Seq(t.data_ptr(), t.stride(0), t.stride(1))
        scan = st.Scan(T, B, n, 1, n, 2, 1, at(rows["u"]), at(rows["dt"]), st.Seq(), at(rows["B"]), at(rows["C"]), A[part].data_ptr(), None, None,
                       ends.data_ptr())
        dB, dC = (torch.full((T, B, n), 7.0, dtype=BF16, device="cuda") for _ in range(2))
        g = st.ScanGradientBuffers(B=at(dB), C=at(dC))
        need = ops.scan_sizes(T, B, n, 1, n)[1]
        work = torch.empty(need, dtype=torch.uint8, device="cuda")
        dy = rows["dy"]
        assert ops._library().sprnn_scan_backward(0, ctypes.byref(scan), ops.Seq(dy.data_ptr(), dy.stride(0), dy.stride(1)), None, kept.data_ptr(),
                                                  ctypes.byref(g), work.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        return dB, dC

    whole = backward(slice(0, C))
    for first in (0, C // 2 - 5, C - some):
        part = slice(first, first + some)
        for got, want in zip(whole, backward(part)):
            assert torch.equal(got[:, :, part], want) and torch.isfinite(want).all() and float(want.abs().max()) > 0
            for b, n in enumerate(ends.tolist()):
                assert (want[n:, b] == 0).all()
    assert not (whole[0] == 7.0).all(dim=2).any()


@pytest.mark.parametrize("T,B,C,N,G,dtype,lengths", slow.CASES)
def test_scans_that_forget_slowly_hold_their_state_in_binary32(T, B, C, N, G, dtype, lengths):
    """Over all elements, not in the worst case: a state that is rounded to 16 bits anywhere along the way is far outside."""
    ops = _ops()
    case, dy, ds = slow.make(T, B, C, N, G, dtype, T)
    want = ref.scan(**_double(case), lengths=lengths, dy=dy.double(), d_state=ds.double())
    dev = {k: v.cuda() for k, v in case.items()}
    args, rest = [dev[k] for k in ("u", "dt", "A", "B", "C")], {k: dev[k] for k in ("D", "z", "dt_bias")}
    rest["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y, s = ops.selective_scan(*args, state=dev["state"], **rest)
    y2, s2, kept = ops.selective_scan(*args, state=dev["state"], keep=True, **rest)
    assert torch.equal(y, y2) and torch.equal(s, s2)
    off = {"y": slow.distance(y, want["y"]) / slow.allowed(case, False, dtype), "state": slow.distance(s, want["state"]) / slow.allowed(case)}
    g = ops.selective_scan_backward(dy.cuda(), *args, kept, d_state=ds.cuda(), **rest)
    for name in g._fields:
        got = getattr(g, name)
        off[name] = slow.distance(got, want[name]) / slow.allowed(case, True, got.dtype)
    print("of the bound: " + ", ".join("%s %.3f" % x for x in off.items()), flush=True)
    assert max(off.values()) <= 1.0, off


@pytest.mark.parametrize("T", [9, 300])
def test_what_lies_behind_a_samples_end_is_neither_used_nor_changed(T):
    """Every operator with lengths: the same bits whatever stands behind the ends, zeros in the outputs there, inputs untouched."""
    ops = _ops()
    B, C, N, K = 4, 70, 16, 4
    ends = [T, T // 2 + 1, 1, 0]
    lengths = torch.tensor(ends, dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(T)
    inputs = {k: torch.randn((T, B, C), generator=gen).to(BF16) for k in ("u", "dt", "z", "dy")}
    inputs.update({k: torch.randn((T, B, 1, N), generator=gen).to(BF16) for k in ("B", "C")})
    A, weight = -torch.rand((C, N), generator=gen).cuda() - 0.1, torch.randn((C, K), generator=gen).cuda()
    runs = []
    for fill in (0.0, float("nan"), float("inf"), torch.finfo(BF16).min):
        own = {k: v.clone() for k, v in inputs.items()}
        for v in own.values():
            for b, n in enumerate(ends):
                v[n:, b] = fill
        dev = {k: v.cuda() for k, v in own.items()}
        y, s, kept = ops.selective_scan(dev["u"], dev["dt"], A, dev["B"], dev["C"], z=dev["z"], lengths=lengths, keep=True)
        g = ops.selective_scan_backward(dev["dy"], dev["u"], dev["dt"], A, dev["B"], dev["C"], kept, z=dev["z"], lengths=lengths)
        c, cs = ops.causal_conv(dev["u"], weight, lengths=lengths)
        dx, dw, _, dcs = ops.causal_conv_backward(dev["dy"], dev["u"], weight, lengths=lengths)
        for b, n in enumerate(ends):
            for out in (y, g.du, g.ddt, g.dz, g.dB, g.dC, c, dx):
                assert (out[n:, b] == 0).all()
        bits = lambda t: t.cpu().view(torch.int16)
        assert all(torch.equal(bits(dev[k]), own[k].view(torch.int16)) for k in own)
        runs.append((y, s, g.du, g.ddt, g.dA, g.dB, g.dC, g.dz, g.dstate, c, cs, dx, dw, dcs))
    for run in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(run, runs[0]))


# T, B, K, R: few rows, tiles with two halves of the slabs, tiles with one, rows without whole pieces
@pytest.mark.parametrize("T,B,K,R", [(1, 8, 256, 300), (20, 8, 640, 5800), (64, 32, 384, 2560), (20, 8, 130, 5800)])
def test_captured_projections_replay_like_eager_ones(T, B, K, R):
    """Every kernel of the projection in a graph, on new inputs and between eager calls."""
    ops = _ops()
    gen = torch.Generator().manual_seed(K)
    e4m3 = lambda *s: torch.randn(s, generator=gen).to(torch.float8_e4m3fn)
    x, w = e4m3(T, B, K).cuda(), e4m3(R, K).cuda()
    xs, ws = torch.rand((T, B, -(-K // 128)), generator=gen).cuda(), torch.rand((-(-R // 128), -(-K // 128)), generator=gen).cuda()
    call = lambda: [ops.project_fp8(x, xs, w, ws, dtype=t) for t in (F32, F16, BF16)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outputs = call()
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(4):
        x.copy_(e4m3(T, B, K))
        xs.copy_(torch.rand(xs.shape, generator=gen))
        want = call()
        for o in outputs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want)), turn
        assert all(torch.isfinite(o.float()).all() for o in (outputs[0], outputs[2]))


def test_the_gradient_of_x_is_the_projection_with_the_weights_transposed():
    """dx = d out w: the gradient of out brought to 8 bits by the caller, w and its scales transposed."""
    ops = _ops()
    T, B, K, R = 7, 9, 272, 400
    gen = torch.Generator().manual_seed(2)
    normal = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)
    w, ws = ref.blocks(normal(R, K) / K ** 0.5, 128, 128)
    d, ds = ref.blocks(normal(T * B, R), 1, 128)
    wt, wst = w.view(torch.uint8).t().contiguous().view(torch.float8_e4m3fn), ws.t().contiguous()
    dx = ops.project_fp8(d.view(T, B, R).cuda(), ds.view(T, B, -1).cuda(), wt.cuda(), wst.cuda())
    # what autograd gives for the dequantised product
    x = normal(T * B, K).requires_grad_()
    full = w.double() * ws.double().repeat_interleave(128, 0)[:R].repeat_interleave(128, 1)[:, :K]
    grad = d.double() * ds.double().repeat_interleave(128, 1)[:, :R]
    (want,) = torch.autograd.grad((x @ full.t() * grad).sum(), [x])
    _close(dx, want.view(T, B, K), ref.project(d, ds, wt, wst, absolute=True).view(T, B, K), 128 + 3 + -(-R // 128) + 2, "dx")


def test_calls_on_tensors_that_require_gradients_say_that_there_are_none():
    import warnings
    ops = _ops()
    x, A = torch.zeros((2, 1, 8), device="cuda"), torch.zeros((8, 4), device="cuda")
    low, one = torch.zeros((2, 1, 1, 4), device="cuda"), torch.ones((2, 1, 1), device="cuda")
    q, eight = torch.zeros((2, 1, 8), dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(8, device="cuda")
    leaf = lambda t: t.clone().requires_grad_()
    calls = [lambda: ops.selective_scan(leaf(x), x, A, low, low), lambda: ops.selective_scan(x, x, leaf(A), low, low),
             lambda: ops.selective_scan(x, x, A, low, low, D=leaf(eight)), lambda: ops.causal_conv(x, leaf(A)),
             lambda: ops.causal_conv(x, A, bias=leaf(eight)), lambda: ops.rms_norm(leaf(x)), lambda: ops.rms_norm(x, leaf(eight)),
             lambda: ops.rms_norm_fp8(x, residual=leaf(x)), lambda: ops.project_fp8(q, one, q[:, 0], one[0], bias=leaf(eight[:2]))]
    for call in calls:
        with pytest.warns(UserWarning, match="have no graph") as said:
            call()
        assert len(said) == 1 and said[0].filename == __file__
        with torch.no_grad(), warnings.catch_warnings():
            warnings.simplefilter("error")
            call()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        ops.selective_scan(leaf(x).detach(), x, A, low, low)
        ops.causal_conv(x, A)
        ops.rms_norm(x, eight)
        ops.project_fp8(q, one, q[:, 0], one[0])


def test_arguments_that_are_no_tensors_are_refused_by_name():
    ops = _ops()
    x, A = torch.zeros((2, 1, 8), device="cuda"), torch.zeros((8, 4), device="cuda")
    low, one = torch.zeros((2, 1, 1, 4), device="cuda"), torch.ones((2, 1, 1), device="cuda")
    q = torch.zeros((2, 1, 8), dtype=torch.float8_e4m3fn, device="cuda")
    for name, call in (("state", lambda v: ops.selective_scan(x, x, A, low, low, state=v)), ("D", lambda v: ops.selective_scan(x, x, A, low, low, D=v)),
                       ("z", lambda v: ops.selective_scan(x, x, A, low, low, z=v)), ("state", lambda v: ops.causal_conv(x, A, state=v)),
                       ("B", lambda v: ops.selective_scan(x, x, A, v, low)), ("C", lambda v: ops.selective_scan(x, x, A, low, v)),
                       ("dt", lambda v: ops.selective_scan(x, v, A, low, low)), ("weight", lambda v: ops.causal_conv(x, v)),
                       ("residual", lambda v: ops.rms_norm(x, residual=v)), ("d_residual", lambda v: ops.rms_norm_backward(x, x, d_residual=v)),
                       ("bias", lambda v: ops.causal_conv(x, A, bias=v)), ("weight", lambda v: ops.rms_norm(x, v)),
                       ("bias", lambda v: ops.project_fp8(q, one, q[:, 0], one[0], bias=v))):
        for wrong in ([0.0] * 8, 1.0, x.cpu().numpy()):
            with pytest.raises(TypeError, match=name):
                call(wrong)
