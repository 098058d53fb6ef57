"""Plain 64-bit forms of the linear layers in 8 bits: codes and scales of a matrix, what they stand for, and the three products.

Written from the definitions in include/adapm.h, on torch tensors in fp64 of any device.  Test infrastructure only; shares
no code with the library.
"""
from __future__ import annotations

import torch

TOP = {"int8": 127.0, "e4m3": 448.0}


def _groups(x: torch.Tensor, group: int):
    """The columns of x that share a scale, one block after the other."""
    return x.split(group or x.shape[1], 1)


def scales_of(x: torch.Tensor, code: str, group: int, pow2: bool) -> torch.Tensor:
    """[rows, groups] in fp64 (values that fp32 holds)."""
    out = []
    for part in _groups(x.double(), group):
        m = part.abs().amax(1)
        s = m / torch.full_like(m, TOP[code])
        if pow2:
            mantissa, power = torch.frexp(s)                      # s = mantissa 2^power, 1/2 <= mantissa < 1
            s = torch.exp2(power.double() - (mantissa == 0.5).double())
            # (m / top may have been rounded up to the power of two that it is just above, or down: settle it by a product)
            s = torch.where(s * TOP[code] < m, 2 * s, s)
            s = torch.where(s / 2 * TOP[code] >= m, s / 2, s)
        else:
            s = s.float().double()
        s = torch.where(m == 0, torch.ones_like(s), s.clamp(min=2.0**-126))
        out.append(torch.where(m.isfinite(), s, torch.full_like(s, float("nan"))))
    return torch.stack(out, 1)


def codes_of(x: torch.Tensor, scales: torch.Tensor, code: str, group: int) -> torch.Tensor:
    """The codes as numbers, in fp64."""
    out = []
    for i, part in enumerate(_groups(x.double(), group)):
        q = part / scales[:, i:i + 1]
        q = torch.round(q) if code == "int8" else q.float().to(torch.float8_e4m3fn).double()
        out.append(torch.where(scales[:, i:i + 1].isnan(), torch.zeros_like(q), q))
    return torch.cat(out, 1)


def decode(codes: torch.Tensor, scales: torch.Tensor, group: int) -> torch.Tensor:
    scales = scales.double().reshape(codes.shape[0], -1)
    return torch.cat([part.double() * scales[:, i:i + 1] for i, part in enumerate(_groups(codes, group))], 1)


def forward(x8, xs, w8, ws) -> torch.Tensor:
    return (x8.double() @ w8.double().T) * xs.double()[:, None] * ws.double()[None, :]


def input_grad(dy, w8, ws) -> torch.Tensor:
    return dy.double() @ decode(w8, ws, 0)


def weight_grad(dy, x8, xs, group: int) -> torch.Tensor:
    return dy.double().T @ decode(x8, xs, group)
