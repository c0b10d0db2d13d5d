"""Beam search over a paged cache, with random weights: prompts go into the cache
once, then every request grows by the best continuations of its beams.

A step is bsm_paged_tables (where the new tokens go); per layer
bsm_paged_write_rotary and bsm_paged_attention; then bsm_beam_select on the logits,
and bsm_paged_reorder, which lets tables, lengths and partly filled pages follow the
selected beams and says which pages are free again.

    python examples/beam_search.py [--steps 32] [--check]

--check recomputes the last layer's last outputs of every beam from its tokens in float64.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2002_07062_gb300 import bsm  # noqa: E402


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=200)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--heads-kv", type=int, default=4)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--page", type=int, default=16)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    n, B, hq, hkv, d, V = a.requests, a.beams, a.heads, a.heads_kv, a.dim, a.vocab
    rows, wide = n * B, (a.heads + 2 * a.heads_kv) * a.dim
    prompts = torch.randint(1, a.prompt + 1, (n,)).tolist()
    width = -(-(a.prompt + a.steps) // a.page)
    pages = rows * (width + 1)          # (a row's copied page is taken before any dropped one is free again)
    i32 = dict(dtype=torch.int32, device="cuda")
    k_cache = torch.zeros((a.layers, pages, a.page, hkv, d), dtype=torch.bfloat16, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    free = torch.randperm(pages, device="cuda", dtype=torch.int32)
    tables, cached = torch.full((rows, width), -1, **i32), torch.zeros(rows, **i32)
    starts, lengths = torch.zeros(rows + 1, **i32), torch.zeros(rows, **i32)
    dropped, info = torch.zeros(rows * width, **i32), torch.zeros(4, dtype=torch.int64, device="cuda")
    angle = torch.arange(a.prompt + a.steps, dtype=torch.float64, device="cuda")[:, None] * \
        10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    rotary = torch.cat([angle.cos(), angle.sin()], 1).float()
    new = lambda *s: torch.randn(s, device="cuda").bfloat16()
    embed = new(V, hq * d)
    weights = [(new(hq * d, wide) * (hq * d) ** -0.5, new(hq * d, hq * d) * (hq * d) ** -0.5) for _ in range(a.layers)]
    head = new(hq * d, V) * (hq * d) ** -0.5
    work = torch.empty(bsm.bsm_paged_workspace_bytes(hq, hkv, d, a.prompt), dtype=torch.uint8, device="cuda")
    work_select = torch.empty(bsm.bsm_beam_select_workspace_bytes(n, B, V, B), dtype=torch.uint8, device="cuda")
    work_reorder = torch.empty(bsm.bsm_paged_reorder_workspace_bytes(n, B, width), dtype=torch.uint8, device="cuda")
    scores = torch.full((n, B), -float("inf"), device="cuda")
    scores[:, 0] = 0.0                  # one beam a request until the prompt's end branches
    history = torch.zeros((rows, a.prompt + a.steps), dtype=torch.int64, device="cuda")
    fresh_h = [p if b == 0 else 0 for p in prompts for b in range(B)]
    ids = []
    for r, m in enumerate(fresh_h):
        history[r, :m] = torch.randint(0, V, (m,), device="cuda")
        ids.append(history[r, :m])
    ids = torch.cat(ids)
    stream = torch.cuda.current_stream()
    worst, t0 = 0.0, None
    for step in range(a.steps):
        fresh, tokens_in = torch.tensor(fresh_h, **i32), len(ids)
        slots = torch.empty(tokens_in, dtype=torch.int64, device="cuda")
        positions, owners = torch.empty((2, tokens_in), **i32)
        bsm.bsm_paged_tables(cached, fresh, free, a.page, tables, starts, lengths, slots, positions, owners, info, stream=stream)
        free = free[int(info[1]):]
        x = embed[ids]
        for layer, (w_in, w_out) in enumerate(weights):
            qkv = (x @ w_in).view(tokens_in, hq + 2 * hkv, d)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            bsm.bsm_paged_write_rotary(q, k, v, q, k_cache[layer], v_cache[layer], slots, positions, rotary, stream=stream)
            out = torch.empty((tokens_in, hq, d), dtype=x.dtype, device="cuda")
            bsm.bsm_paged_attention(q, k_cache[layer], v_cache[layer], out, starts, lengths, tables, max(fresh_h), d ** -0.5,
                                    work, flags=bsm.FLAG_CAUSAL, stream=stream)
            x = x + out.view(tokens_in, hq * d) @ w_out
            x = x / x.float().pow(2).mean(-1, keepdim=True).sqrt().to(x.dtype)
        last = (starts[1:].long() - 1).clamp(min=0)
        if a.check and step == a.steps - 1:
            worst = check(embed, weights, rotary, history, lengths, x[last], hq, hkv, d)
        logits = (x[last] @ head).view(n, B, V)
        best, parents, tokens = torch.empty_like(scores), *torch.empty((2, n, B), **i32)
        bsm.bsm_beam_select(logits, scores, best, parents, tokens, work_select, stream=stream)
        bsm.bsm_paged_reorder(parents, lengths, tables, free, lengths, tables, dropped, info, k_cache, v_cache, work_reorder,
                              stream=stream)
        taken, missing, gone, flags = info.tolist()     # (waits for the device, as reading info above does)
        if flags:
            raise RuntimeError("step does not fit: %d pages missing, flags %d" % (missing, flags))
        free = torch.cat([free[taken:], dropped[:gone]])
        source = (torch.arange(n, device="cuda")[:, None] * B + parents).view(-1).long()
        cached, scores, ids = lengths.clone(), best, tokens.view(-1).long()
        history = history[source]
        history[torch.arange(rows, device="cuda"), lengths.long()] = ids
        fresh_h = [1] * rows
        if step == 0:                   # (the first step loads code and libraries)
            torch.cuda.synchronize()
            t0 = time.perf_counter()
    torch.cuda.synchronize()
    if a.steps > 1:
        print("%d requests of %d beams, %d layers: %.0f tokens/s" % (n, B, a.layers, rows * (a.steps - 1) / (time.perf_counter() - t0)))
    if a.check:
        print("largest error of any last output, relative to the largest: %.2g" % worst)
    assert bsm.bsm_device_status() == 0
    return worst


def check(embed, weights, rotary, history, lengths, got, hq, hkv, d):
    """Every row's last hidden state from its tokens, in float64 but for the roundings between
    layers, against the step's."""
    worst = 0.0
    for r, length in enumerate(lengths.tolist()):
        if length == 0:                 # (a beam that is not in use yet)
            continue
        x = embed[history[r, :length]]
        turn = rotary[:length].double()
        c, s = turn[:, None, :d // 2], turn[:, None, d // 2:]

        def rotate(z):
            lo, hi = z[..., :d // 2], z[..., d // 2:]
            return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)

        for w_in, w_out in weights:
            qkv = (x @ w_in).view(length, hq + 2 * hkv, d).double()
            q, k, v = rotate(qkv[:, :hq]), rotate(qkv[:, hq:hq + hkv]), qkv[:, hq + hkv:]
            k, v = (z.repeat_interleave(hq // hkv, 1) for z in (k, v))
            z = torch.einsum("ihd,jhd->hij", q, k) * d ** -0.5
            z = z.masked_fill(torch.ones(z.shape[1:], dtype=torch.bool, device="cuda").triu(1), -float("inf"))
            out = torch.einsum("hij,jhd->ihd", z.softmax(-1), v).to(x.dtype)
            x = x + out.reshape(length, hq * d) @ w_out
            x = x / x.float().pow(2).mean(-1, keepdim=True).sqrt().to(x.dtype)
        worst = max(worst, float((got[r].double() - x[-1].double()).abs().max() / x[-1].double().abs().max()))
    return worst


if __name__ == "__main__":
    main()
