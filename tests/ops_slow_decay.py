"""Scans whose states forget slowly, and how far a computation in binary32 may be from the definition over all elements.

A step multiplies a state by a = exp(d A) near 1 and adds to it: one exponential (0.31 half steps of binary32 in the root mean
square, and after the compensation of its mean 0.02 one way) and one rounding (0.5), 0.6 half steps together.  A state remembers
1 / (d |A|) steps: errors without a direction add up like the root of half of them (their squares decay twice as fast), those
one way like all.  Four times the first is what a sum of many does not pass.  A gradient has gone through two such recurrences.
"""
import math

import torch

from ops_oracle import EPS, half_step

# T, B, C, N, groups, type, lengths
CASES = [
    (1100, 1, 40, 16, 1, torch.float32, None),
    (2048, 2, 24, 12, 3, torch.float32, [2048, 1400]),
    (700, 2, 33, 40, 1, torch.bfloat16, None),
    (1500, 1, 20, 128, 1, torch.float32, None),
    (1000, 2, 9, 4, 1, torch.float16, [777, 1000]),
    (515, 1, 100, 3, 1, torch.float32, None),
    (4096, 1, 16, 16, 1, torch.float32, None),
    (300, 8, 70, 16, 2, torch.bfloat16, [300, 299, 280, 290, 300, 257, 256, 300]),
]


def make(T, B, C, N, G, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen)
    low = lambda x: x.to(dtype)
    case = dict(u=low(normal(T, B, C)), dt=low(normal(T, B, C) * 0.3), A=-torch.rand((C, N), generator=gen) * 0.8 - 0.2, B=low(normal(T, B, G, N)),
                C=low(normal(T, B, G, N)), D=normal(C), z=low(normal(T, B, C)), dt_bias=torch.full((C,), math.log(math.expm1(3e-3))),
                state=normal(B, C, N))
    return case, low(normal(T, B, C)), normal(B, C, N)


def allowed(case, gradient=False, dtype=torch.float32):
    """|| got - want || / || want ||."""
    d = torch.nn.functional.softplus(case["dt"].double() + case["dt_bias"].double()).mean((0, 1))
    memory = min(case["dt"].shape[0], 1.0 / float((d[:, None] * case["A"].double().abs()).min()))
    own = (4 * 0.6 * math.sqrt(memory / 2) + 0.02 * memory + 10) * EPS
    return (2 if gradient else 1) * own + (half_step(dtype) if dtype != torch.float32 else 0.0)


def distance(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())
