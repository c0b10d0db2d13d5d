"""Paged-cache operators from their definitions: tables and slot maps by plain
loops over requests and tokens, attention in 64 bits, token by token masks.
Shares no code with the library."""
from __future__ import annotations

import numpy as np
import torch


def tables(cached, fresh, free, page, table, n_slots):
    """(table, starts, lengths, slots, positions, owners, info[:3]) of one step."""
    table = np.array(table, np.int64)
    width = table.shape[1]
    free = list(free)
    starts, taken, missing = [0], 0, 0
    slots = np.full(n_slots, -1, np.int64)
    pos_of = np.full(n_slots, -1, np.int64)
    owner = np.full(n_slots, -1, np.int64)
    t = 0
    for r, (c, f) in enumerate(zip(cached, fresh)):
        have = min((c + page - 1) // page, width)
        need = min((c + f + page - 1) // page, width)
        for e in range(have, need):
            if taken < len(free):
                table[r, e] = free[taken]
                taken += 1
            else:
                table[r, e] = -1
                missing += 1
        for p in range(c, c + f):
            if t < n_slots:
                e = p // page
                if e < width and table[r, e] >= 0:
                    slots[t] = table[r, e] * page + p % page
                pos_of[t], owner[t] = p, r
            t += 1
        starts.append(t)
    return table, np.array(starts), np.array(cached) + np.array(fresh), slots, pos_of, owner, (t, taken, missing)


def attention(q, k_cache, v_cache, starts, lengths, tables_, scale, causal, window=0):
    """out, lse and, for error bounds, sum_j p_j |v_j| and the largest
    scale * sum_d |q_d k_d| of every row; float64, on q's device.  starts,
    lengths, tables_ are host sequences."""
    T, hq, d = q.shape
    P, hkv = k_cache.shape[1], k_cache.shape[2]
    g = hq // hkv
    f64 = dict(dtype=torch.float64, device=q.device)
    out = torch.zeros((T, hq, d), **f64)
    lse = torch.full((T, hq), -float("inf"), **f64)
    mass = torch.zeros((T, hq, d), **f64)
    size = torch.zeros((T, hq), **f64)
    for r in range(len(lengths)):
        a, b, L = int(starts[r]), int(starts[r + 1]), int(lengths[r])
        if a == b or L == 0:
            continue
        ids = [int(tables_[r][j // P]) for j in range(0, L, P)]
        k = torch.cat([k_cache[i] for i in ids])[:L].double()
        v = torch.cat([v_cache[i] for i in ids])[:L].double()
        key = torch.arange(L, device=q.device)
        pos = L - (b - a) + torch.arange(b - a, device=q.device)
        see = torch.ones((b - a, L), dtype=torch.bool, device=q.device)
        if causal:
            see = key[None, :] <= pos[:, None]
            if window:
                see = see & (key[None, :] > pos[:, None] - window)
        for h in range(hq):
            x = q[a:b, h].double() @ k[:, h // g].t() * scale
            x = torch.where(see, x, torch.full_like(x, -float("inf")))
            top = x.max(1, keepdim=True).values
            top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
            e = torch.exp(x - top)
            s = e.sum(1, keepdim=True)
            p = e / torch.where(s == 0, torch.ones_like(s), s)
            # (keys no token sees take no part at all, whatever they hold)
            any_ = see.any(0)
            out[a:b, h] = p[:, any_] @ v[any_, h // g]
            mass[a:b, h] = p[:, any_] @ v[any_, h // g].abs()
            lse[a:b, h] = (top + torch.log(s))[:, 0]
            size[a:b, h] = (q[a:b, h].double().abs() @ k[any_, h // g].double().abs().t() * scale).amax(1) \
                if any_.any() else 0.0
    return out, lse, mass, size
