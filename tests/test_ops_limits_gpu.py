"""GPU tests of the operators in paper_1804_10223_amd.ops at the ends of what their header allows: values, strides, sizes.

Tolerances are counted as in test_ops_gpu: roundings on the longest path, times half a step of binary32, times the same sums
over absolute values, plus the rounding of the result to its type.
"""
import pytest
import torch

import ops_oracle as ref
from test_ops_gpu import BF16, F16, F32, TYPES, _close, _ops, _place

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
