"""Rotation by positions from its definition, in 64 bits.  Shares no code with
the library."""
from __future__ import annotations

import torch


def rotary(x, positions, table, interleaved):
    """x [tokens, heads, dim] with its first table.shape[1] columns turned, float64, and the
    size sum |x1 cos| + |x2 sin| of every output; rows of positions outside the table are NaN."""
    h = table.shape[1] // 2
    out, size = x.double().clone(), x.double().abs()
    p = torch.as_tensor(positions, device=x.device).long()
    there = (p >= 0) & (p < table.shape[0])
    rows = table.double()[p[there]]
    z = x[there].double()
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        c, s = rows[:, i, None], rows[:, h + i, None]
        x1, x2 = z[:, :, a], z[:, :, b]
        out[there, :, a], out[there, :, b] = x1 * c - x2 * s, x2 * c + x1 * s
        size[there, :, a] = (x1 * c).abs() + (x2 * s).abs()
        size[there, :, b] = (x2 * c).abs() + (x1 * s).abs()
    out[~there] = float("nan")
    return out, size
