"""Operators of a layer around a selective state space scan, as measurable cases through the public entry points.

Sequences are [T][B][H] like everywhere in this library (T steps, B samples advanced together, H channels, H fastest);
an operator that works on a part of a wider tensor is given the view.  A case is one pass through one operator:

  scan        h_t = exp(d_t A) h_{t-1} + d_t u_t B_t,  y_t = (C_t h_t + D u_t) silu(z_t),  d_t = softplus(dt_t + dt_bias);
              whole prompts (T > 1) and single tokens with their state (T = 1)
  scan_train  the same pass keeping what the backward pass reads, and the backward pass
  conv        depthwise causal convolution over the last few inputs with its SiLU, whole prompts and single tokens
  conv_bwd    its gradients
  norm        root-mean-square norm after the residual's addition, output in the stream's type or in e4m3 with a scale per 128
  norm_bwd    its gradients
  project     product of e4m3 rows (a scale per 128) with e4m3 weights (a scale per 128 x 128), the input projection of a layer

``own`` selects this repository's kernels; the plain forms are written with elementary operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5
LARGEST_E4M3 = 448.0
SMALLEST_AMAX = 2.0 ** -100      # a block of zeros has a scale, too


def _scan(name, T, B, C, N, G=1, type="bf16", gate=True, ragged=False, train=False):
    return {"name": name, "op": "scan_train" if train else "scan", "T": T, "B": B, "C": C, "N": N, "G": G, "type": type,
            "gate": gate, "ragged": ragged}


def _conv(name, T, B, C, K=4, type="bf16", ragged=False, backward=False):
    return {"name": name, "op": "conv_bwd" if backward else "conv", "T": T, "B": B, "C": C, "K": K, "type": type, "ragged": ragged}


def _norm(name, T, B, W, type="bf16", residual="fp32", out="same", backward=False):
    return {"name": name, "op": "norm_bwd" if backward else "norm", "T": T, "B": B, "W": W, "type": type, "residual": residual, "out": out}


def _project(name, T, B, K, R, type="fp32", bias=True):
    return {"name": name, "op": "project", "T": T, "B": B, "K": K, "R": R, "type": type, "bias": bias}


def listed():
    return [
        # the next token of a few samples: the state is read and written once, latency counts
        _scan("scan_token_b4", 1, 4, 1152, 16),
        # one long prompt on its own: few channels, a long axis
        _scan("scan_prompt_b1", 4096, 1, 2304, 16),
        # a full batch of prompts of unequal length on a wide layer
        _scan("scan_batch_b8_ragged", 2048, 8, 4608, 16, ragged=True),
        # sizes that divide nothing, three groups of B and C, binary32, no gate
        _scan("scan_771_n12_fp32", 333, 5, 771, 12, G=3, type="fp32", gate=False),
        # gradients of an ordinary training batch
        _scan("scan_train_b8", 1024, 8, 2048, 16, train=True),
        # the convolution of a training batch or of prompts; the next token of a full batch; its gradients
        _conv("conv_prompt_b8", 2048, 8, 4608),
        _conv("conv_token_b8", 1, 8, 4608, type="fp16"),
        _conv("conv_train_b8", 1024, 8, 2048, backward=True),
        # norm in front of an 8-bit projection, the residual stream in binary32; gradients, stream in bfloat16
        _norm("norm_8bit_2304", 2048, 8, 2304, out="e4m3"),
        _norm("norm_train_2560", 1024, 8, 2560, residual="bf16", backward=True),
        # an 8-bit projection: the next token of a batch (the weights are all there is to read), and whole prompts
        _project("project_token_b8", 1, 8, 2304, 9216, type="bf16", bias=False),
        _project("project_prompt_b8", 1024, 8, 2304, 9216),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """A layer's width: three of five are multiples of 64."""
    w = _log_uniform(rng, low, high)
    return max(64, w // 64 * 64) if rng.random() < 0.6 else w


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["scan", "scan", "scan_train", "conv", "conv_bwd", "norm", "norm_bwd", "project", "project"])
    type = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    while True:
        T = 1 if op in ("scan", "conv", "norm", "project") and rng.random() < 0.3 else _log_uniform(rng, 2, 4096)
        B = _log_uniform(rng, 1, 64 if T == 1 else 16)
        if op in ("scan", "scan_train"):
            G = rng.choice([1, 1, 1, 2, 4])
            C, N = -(-_width(rng, 128, 5120) // G) * G, rng.choice([16, 16, 16, 8, 12, 5, 32, 64])
            if T * B * C * N <= (2.7e8 if op == "scan_train" else 1.2e9):
                return _scan("", T, B, C, N, G, type, gate=rng.random() < 0.7, ragged=T > 1 and rng.random() < 0.4, train=op == "scan_train")
        elif op in ("conv", "conv_bwd"):
            C = _width(rng, 128, 10240)
            if T * B * C <= (1.7e7 if op == "conv_bwd" else 7.5e7):
                return _conv("", T, B, C, rng.choice([4, 4, 2, 3]), type, ragged=T > 1 and rng.random() < 0.4, backward=op == "conv_bwd")
        elif op in ("norm", "norm_bwd"):
            W = _width(rng, 128, 10240)
            if T * B * W <= (2.1e7 if op == "norm_bwd" else 3.7e7):
                return _norm("", T, B, W, type, rng.choice([type, "fp32"]), "e4m3" if op == "norm" and rng.random() < 0.6 else "same",
                             backward=op == "norm_bwd")
        else:
            K, R = _width(rng, 128, 5120), _width(rng, 128, 10240)
            if float(T) * B * K * R <= 1.7e11:
                return _project("", T, B, K, R, type, bias=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------------------------- inputs

def _lengths(case, gen):
    """Lengths of the samples: the longest fills the call, the others are spread below."""
    if not case["ragged"]:
        return None
    lengths = torch.randint(1, case["T"] + 1, (case["B"],), device="cuda", generator=gen)
    lengths[int(torch.randint(case["B"], (1,), device="cuda", generator=gen))] = case["T"]
    return lengths.int()


def _blocks(x, rows, cols):
    """x [R, K] as e4m3 with a scale per rows x cols block: (q, scales)."""
    R, K = x.shape
    padded = torch.zeros((-(-R // rows) * rows, -(-K // cols) * cols), device="cuda")
    padded[:R, :K] = x
    tiles = padded.view(padded.shape[0] // rows, rows, padded.shape[1] // cols, cols)
    scales = tiles.abs().amax(dim=(1, 3)).clamp_(min=SMALLEST_AMAX) / LARGEST_E4M3
    q = (tiles / scales[:, None, :, None]).view(padded.shape)[:R, :K].contiguous().to(torch.float8_e4m3fn)
    return q, scales.contiguous()


def prepare(case, seed):
    """What a program holds before the call: parameters in binary32, activations in the case's type, state of the samples."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, T, B, type = case["op"], case["T"], case["B"], TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    def uniform(low, high, *shape):
        return torch.rand(shape, device="cuda", generator=gen) * (high - low) + low

    s = {"case": case}
    if op in ("scan", "scan_train"):
        C, N, G = case["C"], case["N"], case["G"]
        s["u"] = torch.nn.functional.silu(normal(T, B, C)).to(type)
        s["dt"] = (normal(T, B, C) * 0.5).to(type)
        start = torch.exp(uniform(math.log(1e-3), math.log(1e-1), C))            # step sizes a layer starts with
        s["dt_bias"] = start + torch.log(-torch.expm1(-start))                   # softplus of it is the step size
        s["A"] = -torch.arange(1, N + 1, device="cuda").float() * torch.exp(normal(C, N) * 0.2)
        s["D"] = 1.0 + normal(C) * 0.1
        rank = -(-C // 32)
        low = normal(T, B, rank + 2 * G * N).to(type)                            # one projection gives B, C and the step's factors
        s["B"] = low[:, :, rank:rank + G * N].view(T, B, G, N)
        s["C"] = low[:, :, rank + G * N:].view(T, B, G, N)
        s["z"] = normal(T, B, 2 * C).to(type)[:, :, C:] if case["gate"] else None   # the other half of the input projection
        s["state"] = normal(B, C, N) * 0.5
        s["lengths"] = _lengths(case, gen)
        if op == "scan_train":
            s["dy"] = normal(T, B, C).to(type)
            s["d_state"] = normal(B, C, N) * 0.1
    elif op in ("conv", "conv_bwd"):
        C, K = case["C"], case["K"]
        s["x"] = normal(T, B, 2 * C).to(type)[:, :, :C]                          # one half of the input projection
        s["weight"] = uniform(-1.0, 1.0, C, K) / math.sqrt(K)
        s["bias"] = uniform(-1.0, 1.0, C) / math.sqrt(K)
        s["state"] = normal(K - 1, B, C).to(type)
        s["lengths"] = _lengths(case, gen)
        if op == "conv_bwd":
            s["dy"] = normal(T, B, C).to(type)
            s["d_state"] = (normal(K - 1, B, C) * 0.1).to(type)
    elif op in ("norm", "norm_bwd"):
        W = case["W"]
        s["x"] = normal(T, B, W).to(type)
        s["residual"] = (normal(T, B, W) * 2.0).to(TYPES[case["residual"]])
        s["weight"] = 1.0 + normal(W) * 0.2
        if op == "norm_bwd":
            s["dy"] = normal(T, B, W).to(type)
            s["d_residual"] = normal(T, B, W).to(TYPES[case["residual"]])        # what comes back along the residual stream
    else:
        K, R = case["K"], case["R"]
        q, s["scales"] = _blocks(normal(T * B, K), 1, 128)
        s["q"] = q.view(T, B, K)
        s["scales"] = s["scales"].view(T, B, -1)
        s["w"], s["w_scales"] = _blocks(normal(R, K) / math.sqrt(K), 128, 128)
        s["bias"] = normal(R) * 0.1 if case["bias"] else None
    return s


# ----------------------------------------------------------------------------------------------------------- plain forms

def _prefix(a, x, h):
    """h_t = a_t h_{t-1} + x_t along the first axis from h, by doubling the span of every partial result."""
    x = torch.cat([(x[0] + a[0] * h)[None], x[1:]])
    span = 1
    while span < x.shape[0]:
        x = torch.cat([x[:span], x[span:] + a[span:] * x[:-span]])
        a = torch.cat([a[:span], a[span:] * a[:-span]])
        span *= 2
    return x


def _inside(lengths, T, like):
    """[T, B, 1] truth values: the step is one of the sample's own."""
    if lengths is None:
        return torch.ones((T, 1, 1), dtype=torch.bool, device=like.device)
    return (torch.arange(T, device=like.device)[:, None] < lengths[None, :])[:, :, None]


def _softplus(v):
    return torch.where(v > 20.0, v, torch.log1p(torch.exp(torch.clamp(v, max=20.0))))


def _scan_terms(s):
    """Inputs in 32 bits with nothing behind a sample's end; per state a = exp(d A) and the inputs of the recurrence."""
    C, G = s["case"]["C"], s["case"]["G"]
    inside = _inside(s["lengths"], s["u"].shape[0], s["u"])
    zero = torch.zeros((), device="cuda")
    u = torch.where(inside, s["u"].float(), zero)
    v = s["dt"].float() + s["dt_bias"]
    d = torch.where(inside, _softplus(v), zero)
    Bn = torch.where(inside[..., None], s["B"].float(), zero).repeat_interleave(C // G, dim=2)
    Cn = torch.where(inside[..., None], s["C"].float(), zero).repeat_interleave(C // G, dim=2)
    a = torch.exp(d[..., None] * s["A"])
    return inside, u, v, d, Bn, Cn, a


def _scan_plain(s):
    inside, u, v, d, Bn, Cn, a = _scan_terms(s)
    h = _prefix(a, (d * u)[..., None] * Bn, s["state"])
    y = (h * Cn).sum(dim=3) + s["D"] * u
    if s["z"] is not None:
        z = torch.where(inside, s["z"].float(), torch.zeros((), device="cuda"))
        y = y * z / (1.0 + torch.exp(-z))
    return y.to(s["u"].dtype), h[-1].contiguous()


def _scan_train_plain(s):
    case, type = s["case"], s["u"].dtype
    T, B, C, N, G = case["T"], case["B"], case["C"], case["N"], case["G"]
    zero = torch.zeros((), device="cuda")
    inside, u, v, d, Bn, Cn, a = _scan_terms(s)
    h = _prefix(a, (d * u)[..., None] * Bn, s["state"])
    before = torch.cat([s["state"][None], h[:-1]])
    dy = torch.where(inside, s["dy"].float(), zero)
    y, dz = (h * Cn).sum(dim=3) + s["D"] * u, None
    if s["z"] is not None:
        z = torch.where(inside, s["z"].float(), zero)
        sig = 1.0 / (1.0 + torch.exp(-z))
        dz = (dy * y * sig * (1.0 + z * (1.0 - sig))).to(type)
        y, dy = y * z * sig, dy * z * sig
    # g_t = C_t dy_t + a_{t+1} g_{t+1}: the same recurrence from the end
    g = dy[..., None] * Cn
    g = torch.cat([g[:-1], (g[-1] + s["d_state"])[None]])
    after = torch.cat([torch.ones_like(a[:1]), a[1:].flip(0)])
    g = _prefix(after, g.flip(0), torch.zeros_like(s["state"])).flip(0)
    gB = (g * Bn).sum(dim=3)
    through = g * a * before
    dd = u * gB + (through * s["A"]).sum(dim=3)
    dv = torch.where(inside, dd * torch.where(v > 20.0, torch.ones_like(v), 1.0 / (1.0 + torch.exp(-v))), zero)
    dB = (g * (d * u)[..., None]).view(T, B, G, C // G, N).sum(dim=3)
    dC = (h * dy[..., None]).view(T, B, G, C // G, N).sum(dim=3)
    return (y.to(type), h[-1].contiguous(),
            torch.where(inside, d * gB + s["D"] * dy, zero).to(type), dv.to(type), (through * d[..., None]).sum(dim=(0, 1)),
            torch.where(inside[..., None], dB, zero).to(type), torch.where(inside[..., None], dC, zero).to(type),
            (dy * u).sum(dim=(0, 1)), dz, dv.sum(dim=(0, 1)), a[0] * g[0])


def _conv_terms(s):
    """The inputs behind the state's (zeros behind a sample's end), and the sums before the activation."""
    K, T = s["case"]["K"], s["x"].shape[0]
    inside = _inside(s["lengths"], T, s["x"])
    zero = torch.zeros((), device="cuda")
    x = torch.cat([s["state"].float(), torch.where(inside, s["x"].float(), zero)])
    windows = x.unfold(0, K, 1)                                                  # [T, B, C, K]
    return inside, x, windows, (windows * s["weight"]).sum(dim=3) + s["bias"]


def _last(s, values):
    """The K - 1 rows of values [K - 1 + T, B, C] that end with each sample's last input."""
    K, T, B = s["case"]["K"], s["case"]["T"], s["case"]["B"]
    ends = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"].long()
    return (ends[None, :] + torch.arange(K - 1, device="cuda")[:, None])[:, :, None].expand(K - 1, B, values.shape[2])


def _conv_plain(s):
    inside, x, _, p = _conv_terms(s)
    y = torch.where(inside, p / (1.0 + torch.exp(-p)), torch.zeros((), device="cuda"))
    return y.to(s["x"].dtype), x.gather(0, _last(s, x)).to(s["x"].dtype)


def _conv_bwd_plain(s):
    K, T, type = s["case"]["K"], s["case"]["T"], s["x"].dtype
    inside, x, windows, p = _conv_terms(s)
    sig = 1.0 / (1.0 + torch.exp(-p))
    g = torch.where(inside, s["dy"].float() * sig * (1.0 + p * (1.0 - sig)), torch.zeros((), device="cuda"))
    pad = torch.zeros_like(g[:1]).expand(K - 1, -1, -1)
    dx = (torch.cat([pad, g, pad]).unfold(0, K, 1) * s["weight"].flip(1)).sum(dim=3)   # [K - 1 + T, B, C], the state's first
    dx = dx.scatter_add(0, _last(s, dx), s["d_state"].float())
    return dx[K - 1:].to(type), (g[..., None] * windows).sum(dim=(0, 1)), g.sum(dim=(0, 1)), dx[:K - 1].to(type)


def _norm_plain(s):
    r = (s["x"].float() + s["residual"].float()).to(s["residual"].dtype)
    f = r.float()
    y = f * torch.rsqrt((f * f).mean(dim=2, keepdim=True) + EPS) * s["weight"]
    if s["case"]["out"] != "e4m3":
        return y.to(s["x"].dtype), r
    T, B, W = y.shape
    blocks = -(-W // 128)
    tiles = torch.cat([y, y.new_zeros((T, B, blocks * 128 - W))], dim=2).view(T, B, blocks, 128)
    scales = tiles.abs().amax(dim=3).clamp(min=SMALLEST_AMAX) / LARGEST_E4M3
    return (tiles / scales[..., None]).view(T, B, blocks * 128)[..., :W].to(torch.float8_e4m3fn), scales, r


def _norm_bwd_plain(s):
    """Gradients of the sum x + residual (its rows as the forward pass stored them are s["residual"]) and of the weight."""
    f, dy = s["residual"].float(), s["dy"].float()
    rstd = torch.rsqrt((f * f).mean(dim=2, keepdim=True) + EPS)
    n, dn = f * rstd, dy * s["weight"]
    dr = rstd * (dn - n * (dn * n).mean(dim=2, keepdim=True)) + s["d_residual"].float()
    return dr.to(s["residual"].dtype), (dy * n).sum(dim=(0, 1))


def _project_plain(s):
    T, B, K = s["q"].shape
    x = s["q"].float() * s["scales"].repeat_interleave(128, dim=2)[..., :K]
    w = s["w"].float() * s["w_scales"].repeat_interleave(128, dim=0)[:s["w"].shape[0]].repeat_interleave(128, dim=1)[:, :K]
    y = (x.view(T * B, K) @ w.t()).view(T, B, -1)
    return (y if s["bias"] is None else y + s["bias"]).to(TYPES[s["case"]["type"]])


_PLAIN = {"scan": _scan_plain, "scan_train": _scan_train_plain, "conv": _conv_plain, "conv_bwd": _conv_bwd_plain,
          "norm": _norm_plain, "norm_bwd": _norm_bwd_plain, "project": _project_plain}


# ------------------------------------------------------------------------------------------------- this library's kernels

def _run_own(s):
    from paper_1804_10223_amd import ops
    case = s["case"]
    op = case["op"]
    if op == "scan":
        return ops.selective_scan(s["u"], s["dt"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"],
                                  state=s["state"], lengths=s["lengths"])
    if op == "scan_train":
        y, state, kept = ops.selective_scan(s["u"], s["dt"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"],
                                            state=s["state"], lengths=s["lengths"], keep=True)
        return (y, state) + tuple(ops.selective_scan_backward(
            s["dy"], s["u"], s["dt"], s["A"], s["B"], s["C"], kept, D=s["D"], z=s["z"], dt_bias=s["dt_bias"],
            lengths=s["lengths"], d_state=s["d_state"]))
    if op == "conv":
        return ops.causal_conv(s["x"], s["weight"], s["bias"], state=s["state"], lengths=s["lengths"])
    if op == "conv_bwd":
        return ops.causal_conv_backward(s["dy"], s["x"], s["weight"], s["bias"], state=s["state"], lengths=s["lengths"],
                                        d_state=s["d_state"])
    if op == "norm":
        if case["out"] == "e4m3":
            return ops.rms_norm_fp8(s["x"], s["weight"], eps=EPS, residual=s["residual"])
        return ops.rms_norm(s["x"], s["weight"], eps=EPS, residual=s["residual"])
    if op == "norm_bwd":
        return ops.rms_norm_backward(s["dy"], s["residual"], s["weight"], eps=EPS, d_residual=s["d_residual"])
    return ops.project_fp8(s["q"], s["scales"], s["w"], s["w_scales"], s["bias"], dtype=TYPES[case["type"]])


def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["case"]["op"]](state)


# --------------------------------------------------------------------------------------------------------------- the work

def work(case):
    """Least bytes (each input read once, each output written once) and operations (an exponential counts as one)."""
    op, T, B = case["op"], case["T"], case["B"]
    e = 4 if case["type"] == "fp32" else 2
    if op in ("scan", "scan_train"):
        C, N, G = case["C"], case["N"], case["G"]
        steps, gate = T * B * C, 1 if case["gate"] else 0
        low = 2 * T * B * G * N * e
        fixed = 4 * C * (N + 2) + 4 * B * C * N
        if op == "scan":
            return {"bytes": steps * e * (3 + gate) + low + fixed + 4 * B * C * N, "flops": steps * N * 7}
        return {"bytes": steps * e * (6 + 3 * gate) + 2 * low + 2 * fixed + 8 * B * C * N, "flops": steps * N * 27}
    if op in ("conv", "conv_bwd"):
        C, K = case["C"], case["K"]
        values, fixed = T * B * C, 4 * C * (K + 1) + e * (K - 1) * B * C
        if op == "conv":
            return {"bytes": 2 * values * e + fixed + e * (K - 1) * B * C, "flops": values * (2 * K + 4)}
        return {"bytes": 3 * values * e + 2 * fixed + e * (K - 1) * B * C, "flops": values * (6 * K + 8)}
    if op in ("norm", "norm_bwd"):
        W, r = case["W"], 4 if case["residual"] == "fp32" else 2
        values = T * B * W
        if op == "norm":
            out = values + 4 * T * B * -(-W // 128) if case["out"] == "e4m3" else values * e
            return {"bytes": values * (e + 2 * r) + out + 4 * W, "flops": values * 6}
        return {"bytes": values * (e + 3 * r) + 8 * W, "flops": values * 12}
    K, R = case["K"], case["R"]
    blocks = -(-K // 128)
    return {"bytes": T * B * (K + 4 * blocks) + R * K + 4 * blocks * -(-R // 128) + T * B * R * e, "flops": 2.0 * T * B * K * R}


# -------------------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_scan(s, u, dt, A, Bm, Cm, D, z, bias, state):
    """One step after the other; inputs in 64 bits.  Returns y and the state behind each sample's last step."""
    case = s["case"]
    T, B, C, N, G = case["T"], case["B"], case["C"], case["N"], case["G"]
    ends = [T] * B if s["lengths"] is None else s["lengths"].tolist()
    ends = torch.tensor(ends, device="cuda")
    h, rows = state, []
    Ag, Dg = A.view(G, C // G, N), D.view(G, C // G)
    for t in range(T):
        alive = (t < ends).view(B, 1, 1)
        step = torch.nn.functional.softplus(dt[t] + bias).view(B, G, C // G, 1)
        ut = u[t].view(B, G, C // G, 1)
        new = (torch.exp(step * Ag) * h.view(B, G, C // G, N) + step * ut * Bm[t][:, :, None, :])
        yt = (new * Cm[t][:, :, None, :]).sum(-1) + Dg * ut[..., 0]
        h = torch.where(alive, new.reshape(B, C, N), h)
        yt = yt.reshape(B, C)
        if z is not None:
            yt = yt * torch.nn.functional.silu(z[t])
        rows.append(torch.where(alive[..., 0], yt, torch.zeros_like(yt)))
    return torch.stack(rows), h


def exact(case, seed):
    s = prepare(case, seed)
    op, T, B = case["op"], case["T"], case["B"]
    if op in ("scan", "scan_train"):
        names = ["u", "dt", "A", "B", "C", "D", "z", "dt_bias", "state"]
        if op == "scan":
            v = [None if s[k] is None else s[k].double() for k in names]
            return _exact_scan(s, *v)
        if T * B * case["C"] * case["N"] > 4e8:
            return None
        v = [None if s[k] is None else s[k].double().requires_grad_() for k in names]
        y, h = _exact_scan(s, *v)
        loss = (y * s["dy"].double()).sum() + (h * s["d_state"].double()).sum()
        grads = iter(torch.autograd.grad(loss, [x for x in v if x is not None]))
        return (y.detach(), h.detach()) + tuple(None if x is None else next(grads) for x in v)
    if op in ("conv", "conv_bwd"):
        K = case["K"]
        ends = [T] * B if s["lengths"] is None else s["lengths"].tolist()
        back = op == "conv_bwd"
        x, w, b, st = [s[k].double().requires_grad_(back) for k in ("x", "weight", "bias", "state")]
        line = torch.cat([st, x])
        p = b + sum(line[k:k + T] * w[:, k] for k in range(K))
        keep = torch.tensor([[t < n for n in ends] for t in range(T)], device="cuda")[:, :, None]
        y = torch.where(keep, torch.nn.functional.silu(p), torch.zeros_like(p))
        h = torch.stack([line[ends[i]:ends[i] + K - 1, i] for i in range(B)], dim=1)
        if not back:
            return y, h
        return torch.autograd.grad((y * s["dy"].double()).sum() + (h * s["d_state"].double()).sum(), (x, w, b, st))
    if op in ("norm", "norm_bwd"):
        W = case["W"]
        if op == "norm":
            r = s["x"].double() + s["residual"].double()
            y = r / torch.sqrt(r.pow(2).sum(2, keepdim=True) / W + EPS) * s["weight"].double()
            if case["out"] != "e4m3":
                return y, r
            q, scales = torch.empty_like(y), []
            for k in range(0, W, 128):
                top = y[..., k:k + 128].abs().max(dim=2).values
                scales.append(torch.maximum(top, torch.full_like(top, SMALLEST_AMAX)) / LARGEST_E4M3)
                q[..., k:k + 128] = y[..., k:k + 128] / scales[-1][..., None]
            return q, torch.stack(scales, dim=2), r
        r, w = s["residual"].double().requires_grad_(), s["weight"].double().requires_grad_()
        y = r / torch.sqrt(r.pow(2).sum(2, keepdim=True) / W + EPS) * w
        return torch.autograd.grad((y * s["dy"].double()).sum() + (r * s["d_residual"].double()).sum(), (r, w))
    K, R = case["K"], case["R"]
    x, w = s["q"].double().view(T * B, K), s["w"].double()
    y = torch.zeros((T * B, R), dtype=torch.float64, device="cuda")
    for k in range(0, K, 128):
        column = s["w_scales"][:, k // 128].double().repeat_interleave(128)[:R]
        y += (x[:, k:k + 128] @ w[:, k:k + 128].t()) * s["scales"].view(T * B, -1)[:, k // 128].double()[:, None] * column
    return (y if s["bias"] is None else y + s["bias"].double()).view(T, B, R)
