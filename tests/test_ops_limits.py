"""CPU: what the C entry points of the sequence operators refuse at the ends of their ranges (nothing here reaches a GPU), and
what the GPU tests' bound for slow scans tells apart."""
import ctypes

import pytest
import torch

import ops_oracle as ref
import ops_slow_decay as slow
import ops_structures as st
from paper_1804_10223_amd import binding, ops
from test_ops_oracle import AT, _own, _scan_arguments, _seq


@pytest.mark.parametrize("name", ["u", "dt", "z", "B", "C", "y"])
def test_two_steps_of_a_scan_are_at_most_2_25_elements_apart(name):
    lib, far = ops._library(), _seq(step=(1 << 25) + 1, sample=8)
    s = _scan_arguments(steps=2, **({} if name == "y" else {name: far}))
    y = far if name == "y" else _seq()
    assert lib.sprnn_scan_forward(0, ctypes.byref(s), None, y, None, None, None, 0, None) == binding.SPRNN_ERR_INVALID
    g = st.ScanGradientBuffers(u=_own(y))
    assert lib.sprnn_scan_backward(0, ctypes.byref(s), _seq(), None, AT, ctypes.byref(g), AT, 1 << 40, None) == binding.SPRNN_ERR_INVALID


def _recurrence(case, every=0, to=None, chained=0.0):
    """y and the last state in binary32; every `every` steps the state is rounded to `to`, or decays by a sum of d that is off by
    the factor `chained`."""
    A, h, rows = case["A"], case["state"], []
    d = torch.nn.functional.softplus(case["dt"].float() + case["dt_bias"])
    groups = case["B"].shape[2]
    spread = lambda x: x.float().repeat_interleave(A.shape[0] // groups, dim=2)
    Bn, Cn, u, z = spread(case["B"]), spread(case["C"]), case["u"].float(), case["z"].float()
    for t in range(u.shape[0]):
        if every and t and t % every == 0:
            if to is not None:
                h = h.to(to).float()
            if chained:
                h = h * torch.exp(chained * d[t - every:t].sum(0)[..., None] * A)
        h = torch.exp(d[t][..., None] * A) * h + (d[t] * u[t])[..., None] * Bn[t]
        rows.append((h * Cn[t]).sum(-1) + case["D"] * u[t])
    return torch.stack(rows) * z * torch.sigmoid(z), h


@pytest.mark.parametrize("T,B,C,N,G,dtype,lengths", [c for c in slow.CASES if c[0] * c[1] <= 1500 and c[6] is None])
def test_the_bound_of_slow_scans_tells_a_rounded_state_from_binary32(T, B, C, N, G, dtype, lengths):
    case, _, _ = slow.make(T, B, C, N, G, dtype, T)
    want = ref.scan(**{k: v.double() for k, v in case.items()})
    most = slow.allowed(case)
    y, h = _recurrence(case)
    assert slow.distance(y, want["y"]) <= most and slow.distance(h, want["state"]) <= most
    for every, to, chained in ((8, torch.bfloat16, 0.0), (64, torch.bfloat16, 0.0), (256, torch.bfloat16, 0.0), (256, torch.float16, 0.0), (64, None, 1e-3)):
        y, h = _recurrence(case, every, to, chained)
        assert slow.distance(y, want["y"]) > most and slow.distance(h, want["state"]) > most, (every, to, chained)
