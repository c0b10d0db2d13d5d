"""Rotation by positions and beam selection from their definitions, in 64 bits.
Shares no code with the library."""
from __future__ import annotations

import math

import numpy as np
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


def select(logits, scores, keep, ended=None, end_token=0):
    """(values, parents, tokens) [n, keep] of the best continuations: float64 numpy logits
    [n, beams, vocab], scores [n, beams].  -inf, -1, -1 where there are no more."""
    n, B, V = logits.shape
    values = np.full((n, keep), -np.inf)
    parents = np.full((n, keep), -1, np.int64)
    tokens = np.full((n, keep), -1, np.int64)
    for r in range(n):
        cand = []
        for b in range(B):
            s = float(scores[r, b])
            if not math.isfinite(s):
                continue
            if ended is not None and ended[r, b]:
                cand.append((s, b, end_token))
                continue
            x = logits[r, b].astype(np.float64)
            if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all():
                continue
            m = x.max()
            lse = np.log(np.exp(x - m).sum())
            # the row's best by (logit, then lowest token); the beams compete by value
            best = np.lexsort((np.arange(V), -x))[:keep]
            cand += [(s + ((x[v] - m) - lse), b, int(v)) for v in best if x[v] > -np.inf]
        cand.sort(key=lambda c: (-c[0], c[1], c[2]))
        for i, (v, b, t) in enumerate(cand[:keep]):
            values[r, i], parents[r, i], tokens[r, i] = v, b, t
    return values, parents, tokens
