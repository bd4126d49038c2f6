"""Plain implementations in 64 bits (torch, any device) of the steps between two attention
calls of a decode step, from the definitions in include/daf.h; test infrastructure only.
"""
from __future__ import annotations

import torch

BLOCK = 32
MIN_EXP = -100

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def e2m1_values(codes):
    """[n][k / 2] bytes to [n][k] values."""
    table = torch.tensor(E2M1 + [-x for x in E2M1], dtype=torch.float64, device=codes.device)
    return torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(1)


def scales_of(b):
    """Values of scale bytes."""
    e = torch.exp2(b.double().clamp(27, 247) - 127)
    return torch.where(b == 255, torch.nan, e)


def mx_values(values, scale_bytes):
    """[n][k] code values times their blocks' scales."""
    return values.double() * scales_of(scale_bytes).repeat_interleave(BLOCK, 1)


def linear(a, w, bias=None, residual=None):
    """C and, per element, the sum of the products' magnitudes; a, w: float64."""
    c, size = a @ w.t().contiguous(), a.abs() @ w.abs().t().contiguous()
    if bias is not None:
        c, size = c + bias.double(), size + bias.double().abs()
    if residual is not None:
        c, size = c + residual.double(), size + residual.double().abs()
    return c, size


def rmsnorm(s, w, eps):
    s = s.double()
    return s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * w.double()
