"""The operators of paper_1804_10223_amd.ops from their definitions, in 64 bits, one step after the other (test infrastructure).

``absolute=True`` runs the same sums over absolute values.  Rounding errors of a computation in 32 bits are bounded by the
number of roundings on the longest path from an input to a result, times half a step, times that sum: the tests' tolerances
are such counts.
"""
import torch

EPS = 2.0 ** -24          # half a step of binary32, relative


def half_step(dtype):
    return {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}[dtype]


def smallest(dtype):
    """Half of the smallest step, for results below the normal range."""
    return {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float8_e4m3fn: 2.0 ** -10}[dtype]


def ends_of(lengths, T, B):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


def _inside(ends, T):
    return torch.tensor([[t < n for n in ends] for t in range(T)], dtype=torch.bool).view(T, len(ends))


def _clean(x, inside):
    """Zeros behind the ends, whatever stands there."""
    shape = inside.shape + (1,) * (x.dim() - 2)
    return torch.where(inside.view(shape), x, torch.zeros((), dtype=x.dtype))


def scan(u, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, state=None, lengths=None, dy=None, d_state=None,
         absolute=False):
    """Everything in float64 on the CPU.  Returns a dict: y, state, and with dy the gradients du, ddt, dA, dB, dC, dD, dz,
    ddt_bias, dstate."""
    T, batch, channels = u.shape
    groups, N = B.shape[2], B.shape[3]
    inside = _inside(ends_of(lengths, T, batch), T)
    mag = torch.abs if absolute else (lambda x: x)
    u, dt, B, C = (_clean(x, inside) for x in (u, dt, B, C))
    v = dt if dt_bias is None else dt + dt_bias
    d = _clean(torch.nn.functional.softplus(v, threshold=200.0) if softplus else v, inside)
    slope = torch.sigmoid(v) if softplus else torch.ones_like(v)
    spread = lambda x: mag(x).repeat_interleave(channels // groups, dim=2)
    Bc, Cc, u_ = spread(B), spread(C), mag(u)
    a = torch.exp(d[..., None] * A)
    d_ = mag(d)
    h = torch.zeros((batch, channels, N), dtype=torch.float64) if state is None else mag(state).clone()
    before, after, y = [], [], []
    for t in range(T):
        before.append(h)
        h = a[t] * h + (d_[t] * u_[t])[..., None] * Bc[t]
        after.append(h)
        y.append((h * Cc[t]).sum(-1) + (0.0 if D is None else mag(D) * u_[t]))
    y = torch.stack(y) if T else torch.zeros_like(u)
    raw = y
    if z is not None:
        z = _clean(z, inside)
        s = torch.sigmoid(z)
        y = y * mag(z * s)
    out = {"y": _clean(y, inside), "state": h}
    if dy is None:
        return out
    e = mag(_clean(dy, inside))
    out["dz"] = None
    if z is not None:
        out["dz"] = e * raw * mag(s * (1.0 + z * (1.0 - s)))
        e = e * mag(z * s)
    g = torch.zeros_like(h) if d_state is None else mag(d_state).clone()
    du, dd, dA = torch.zeros_like(u), torch.zeros_like(u), torch.zeros_like(A)
    dB, dC = torch.zeros_like(B), torch.zeros_like(C)
    for t in reversed(range(T)):
        g = g + Cc[t] * e[t][..., None]
        through = g * a[t] * before[t]
        gB = (g * Bc[t]).sum(-1)
        du[t] = d_[t] * gB + (0.0 if D is None else mag(D) * e[t])
        dd[t] = u_[t] * gB + (through * mag(A)).sum(-1)
        dA += (through * d_[t][..., None]).sum(0)
        dB[t] = (g * (d_[t] * u_[t])[..., None]).view(batch, groups, -1, N).sum(2)
        dC[t] = (after[t] * e[t][..., None]).view(batch, groups, -1, N).sum(2)
        g = g * a[t]
    dv = _clean(dd * slope, inside)
    out.update(du=_clean(du, inside), ddt=dv, dA=dA, dB=_clean(dB, inside), dC=_clean(dC, inside),
               dD=None if D is None else (e * u_).sum((0, 1)), ddt_bias=None if dt_bias is None else dv.sum((0, 1)), dstate=g)
    return out


def conv(x, weight, bias=None, silu=True, state=None, lengths=None, dy=None, d_state=None, absolute=False):
    T, batch, channels = x.shape
    K = weight.shape[1]
    ends = ends_of(lengths, T, batch)
    inside = _inside(ends, T)
    mag = torch.abs if absolute else (lambda v: v)
    x = _clean(x, inside)
    past = torch.zeros((K - 1, batch, channels), dtype=torch.float64) if state is None else state
    line = torch.cat([past, x])
    b = torch.zeros(channels, dtype=torch.float64) if bias is None else bias
    p = torch.zeros_like(x) + b
    p_mag = torch.zeros_like(x) + b.abs()
    for k in range(K):
        p = p + line[k:k + T] * weight[:, k]
        p_mag = p_mag + (line[k:k + T] * weight[:, k]).abs()
    s = torch.sigmoid(p)
    y = p * s if silu else p
    # |y| can be far below what it is the difference of
    out = {"y": _clean(torch.maximum(p_mag, y.abs()) if absolute else y, inside)}
    out["state"] = torch.stack([line[n:n + K - 1, i] for i, n in enumerate(ends)], dim=1) if K > 1 else past
    if dy is None:
        return out
    # slope of silu: at most 1.1; an error of p moves it by at most half of that error
    slope = s * (1.0 + p * (1.0 - s)) if silu else torch.ones_like(p)
    if absolute:
        slope = 1.1 + p_mag if silu else torch.ones_like(p)
    g = mag(_clean(dy, inside)) * slope
    d_line = torch.zeros_like(line)
    dw = torch.zeros_like(weight)
    for k in range(K):
        d_line[k:k + T] += g * mag(weight[:, k])
        dw[:, k] = (g * mag(line[k:k + T])).sum((0, 1))
    if d_state is not None:
        for i, n in enumerate(ends):
            d_line[n:n + K - 1, i] += mag(d_state[:, i])
    out.update(dx=d_line[K - 1:], dweight=dw, dbias=None if bias is None else g.sum((0, 1)), dstate=d_line[:K - 1])
    return out


def norm(r, weight=None, eps=1e-5):
    y = r / torch.sqrt((r * r).mean(-1, keepdim=True) + eps)
    return y if weight is None else y * weight


def norm_backward(dy, r, weight=None, eps=1e-5, d_residual=None, absolute=False):
    mag = torch.abs if absolute else (lambda v: v)
    rs = 1.0 / torch.sqrt((r * r).mean(-1, keepdim=True) + eps)
    n, g = mag(r) * rs, mag(dy) * (1.0 if weight is None else mag(weight))
    along = n * (g * n).mean(-1, keepdim=True)
    dr = rs * (g + along if absolute else g - along) + (0.0 if d_residual is None else mag(d_residual))
    return dr, None if weight is None else (mag(dy) * n).reshape(-1, r.shape[-1]).sum(0)


def blocks(x, rows, cols):
    """float64 [R, K] -> (e4m3 of it with a scale per rows x cols block, float32 scales)."""
    R, K = x.shape
    scales = torch.zeros((-(-R // rows), -(-K // cols)), dtype=torch.float64)
    q = torch.zeros((R, K), dtype=torch.float64)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            part = x[i * rows:(i + 1) * rows, j * cols:(j + 1) * cols]
            scale = torch.tensor(max(float(part.abs().max()), 2.0 ** -100) / 448.0).float()
            scales[i, j] = scale.double()
            q[i * rows:(i + 1) * rows, j * cols:(j + 1) * cols] = (part / scale.double()).clamp(-448.0, 448.0)
    return q.float().to(torch.float8_e4m3fn), scales.float()


def project(q, x_scales, w, w_scales, bias=None, absolute=False):
    """q [M, K], x_scales [M, ceil(K / 128)], w [R, K], w_scales [ceil(R / 128), ceil(K / 128)]."""
    M, K = q.shape
    R = w.shape[0]
    mag = torch.abs if absolute else (lambda v: v)
    x = mag(q.double() * x_scales.double().repeat_interleave(128, dim=1)[:, :K])
    wd = mag(w.double() * w_scales.double().repeat_interleave(128, dim=0)[:R].repeat_interleave(128, dim=1)[:, :K])
    y = x @ wd.t()
    return y if bias is None else y + mag(bias.double())
