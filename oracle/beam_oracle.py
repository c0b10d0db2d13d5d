"""Rotation by positions, beam selection and beam reordering from their
definitions, by plain loops and in 64 bits.  Shares no code with the library."""
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


def reorder(parents, lengths, tables, free, page):
    """New (lengths, tables as {(row, column): page}, copies [(source, page, tokens)],
    missing, dropped) for parents [n][beams], lengths and tables of n * beams rows."""
    n, B = len(parents), len(parents[0])
    need = lambda L: -(-L // page)
    new_len, new_tab, copies, missing, dropped = [], {}, [], 0, []
    taken = 0
    for r in range(n):
        held = set()
        rows = []
        for i in range(B):
            p = parents[r][i]
            L = lengths[r * B + p] if 0 <= p < B else 0
            row = [int(tables[r * B + p][c]) for c in range(need(L))] if L else []
            if L % page and row[-1] >= 0:
                if row[-1] in held:
                    if taken < len(free):
                        copies.append((row[-1], int(free[taken]), L % page))
                        row[-1] = int(free[taken])
                        taken += 1
                    else:
                        row[-1] = -1
                        missing += 1
                else:
                    held.add(row[-1])
            rows.append(row)
            new_len.append(L)
            for c, v in enumerate(row):
                new_tab[r * B + i, c] = v
        most = max(need(lengths[r * B + b]) for b in range(B))
        for c in range(most):
            now = {row[c] for row in rows if c < len(row)}
            seen = set()
            for b in range(B):
                if c < need(lengths[r * B + b]):
                    e = int(tables[r * B + b][c])
                    if e >= 0 and e not in now and e not in seen:
                        dropped.append(e)
                    seen.add(e)
    return new_len, new_tab, copies, missing, dropped
