"""A server's steps over a paged cache, with random weights: prompts come in
chunks, then every request grows by one token a step.

Per step, bsm_paged_tables gives new pages to the requests and says where every
new token goes; per layer, bsm_paged_write stores the new keys and values and
bsm_paged_attention attends over all of them.  Lengths, tables and slots stay on
the device; the host knows only how many tokens it put into the step.

    python examples/paged_serving.py [--steps 32] [--check]

--check recomputes every request's outputs from its whole history in float64.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2002_07062_gb300 import bsm  # noqa: E402


class PagedCache:
    """Keys and values of `layers` layers in one pool of pages."""

    def __init__(self, layers, pages, page, heads_kv, dim, max_requests, width, dtype=torch.bfloat16):
        self.page = page
        self.k = torch.zeros((layers, pages, page, heads_kv, dim), dtype=dtype, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.free = torch.randperm(pages, device="cuda", dtype=torch.int32)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.tables = torch.full((max_requests, width), -1, **i32)
        self.cached = torch.zeros(max_requests, **i32)
        self.starts, self.lengths = torch.zeros(max_requests + 1, **i32), torch.zeros(max_requests, **i32)
        self.info = torch.zeros(4, dtype=torch.int64, device="cuda")

    def begin(self, fresh, tokens):
        """Places `tokens` new tokens, fresh[r] of request r; returns their slots and positions."""
        slots = torch.empty(tokens, dtype=torch.int64, device="cuda")
        pos, owner = torch.empty((2, tokens), dtype=torch.int32, device="cuda")
        bsm.bsm_paged_tables(self.cached, fresh, self.free, self.page, self.tables, self.starts, self.lengths, slots, pos,
                             owner, self.info, stream=torch.cuda.current_stream())
        return slots, pos, owner

    def commit(self, fresh):
        """The step's tokens are in the cache (the one place that waits for the device)."""
        tokens, taken, missing, flags = self.info.tolist()
        if flags:
            raise RuntimeError("step does not fit: %d pages missing, flags %d" % (missing, flags))
        self.free = self.free[taken:]
        self.cached += fresh


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--chunk", type=int, default=256)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--heads-kv", type=int, default=4)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--page", type=int, default=16)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    n, hq, hkv, d = a.requests, a.heads, a.heads_kv, a.dim
    prompts = torch.randint(max(1, a.prompt // 3), a.prompt + 1, (n,)).tolist()
    width = -(-(a.prompt + a.steps) // a.page)
    cache = PagedCache(a.layers, n * width, a.page, hkv, d, n, width)
    wide = (hq + 2 * hkv) * d
    weights = [(torch.randn(hq * d, wide, device="cuda").bfloat16() * (hq * d) ** -0.5,
                torch.randn(hq * d, hq * d, device="cuda").bfloat16() * (hq * d) ** -0.5) for _ in range(a.layers)]
    ws = torch.empty(bsm.bsm_paged_workspace_bytes(hq, hkv, d, a.chunk), dtype=torch.uint8, device="cuda")
    history = [[[] for _ in range(n)] for _ in range(a.layers)]     # (q, k, v, out) of every layer and request
    done = [0] * n
    state = torch.randn(n, hq * d, device="cuda").bfloat16()        # what a request's next single token is made of
    total, t0 = 0, None
    for step in range(a.steps + -(-a.prompt // a.chunk)):
        fresh_h = [min(a.chunk, p - x) if x < p else 1 for p, x in zip(prompts, done)]
        tokens = sum(fresh_h)
        fresh = torch.tensor(fresh_h, dtype=torch.int32, device="cuda")
        ends = torch.tensor(fresh_h).cumsum(0).cuda() - 1
        x = torch.randn(tokens, hq * d, device="cuda").bfloat16()
        x[ends] = state
        slots, _, _ = cache.begin(fresh, tokens)
        for layer, (w_in, w_out) in enumerate(weights):
            qkv = (x @ w_in).view(tokens, hq + 2 * hkv, d)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            bsm.bsm_paged_write(k, v, cache.k[layer], cache.v[layer], slots, stream=torch.cuda.current_stream())
            out = torch.empty((tokens, hq, d), dtype=x.dtype, device="cuda")
            bsm.bsm_paged_attention(q, cache.k[layer], cache.v[layer], out, cache.starts, cache.lengths, cache.tables,
                                    max(fresh_h), d ** -0.5, ws, flags=bsm.FLAG_CAUSAL,
                                    stream=torch.cuda.current_stream())
            if a.check:
                for r, part in enumerate(zip(*(z.split(fresh_h) for z in (q, k, v, out)))):
                    history[layer][r].append([z.clone() for z in part])
            x = x + out.view(tokens, hq * d) @ w_out
            x = x / x.float().pow(2).mean(-1, keepdim=True).sqrt().to(x.dtype)
        state = x[ends]
        cache.commit(fresh)
        done = [y + f for y, f in zip(done, fresh_h)]
        if step:                        # (the first step loads code and libraries)
            total += tokens
        else:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
    torch.cuda.synchronize()
    print("%d requests, %d layers: %.0f tokens/s" % (n, a.layers, total / (time.perf_counter() - t0)))
    if not a.check:
        return 0.0
    worst = 0.0
    for rows in history:
        for r in range(n):
            q, k, v, out = (torch.cat(z).double() for z in zip(*rows[r]))
            k, v = (z.repeat_interleave(hq // hkv, 1) for z in (k, v))
            s = torch.einsum("ihd,jhd->hij", q, k) * d ** -0.5
            s = s.masked_fill(torch.ones(s.shape[1:], dtype=torch.bool, device="cuda").triu(1), -float("inf"))
            ref = torch.einsum("hij,jhd->ihd", s.softmax(-1), v)
            worst = max(worst, float((out - ref).abs().max() / ref.abs().max()))
    print("largest error of any output, relative to the largest output: %.2g" % worst)
    assert bsm.bsm_device_status() == 0
    return worst


if __name__ == "__main__":
    main()
