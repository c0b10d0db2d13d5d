"""The paged-cache operators as they are measured: block tables and slot maps
from request lengths, new keys and values written to their slots, and
attention of new tokens over the cache, alone and as one step.

A case is a dict:
  kind    "tables", "write", "attention" or "step" (the three in turn)
  n       requests; every one has up to `cached` tokens in the cache already
          (uniform from cached_min), `chunks` of them bring up to `new` tokens
          (uniform from new_min), the others one
  page    tokens a page holds
  hq, hkv, d, dtype      query heads, key/value heads, head size, "bf16" or "f16"
  causal, window, lse    the mask, and whether log-sum-exp is returned
  lens_seed              draws the lengths
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16}
_ROWS = 1 << 28          # scores of a plain pass held at once

_MAX_FLOPS = 1.09e12     # a drawn case at most: the largest listed ones'
_MAX_BYTES = 2_200_000_000
_MAX_TOKENS = 1 << 18


def _case(name, kind, n, cached_min, cached, chunks, new_min, new, page, lens_seed, hq=32, hkv=8, d=128, dtype="bf16",
          causal=True, window=0, lse=False, pad=1):
    c = dict(kind=kind, n=n, cached_min=cached_min, cached=cached, chunks=chunks, new_min=new_min, new=new, page=page,
             lens_seed=lens_seed, pad=pad)
    if kind != "tables":
        c.update(hkv=hkv, d=d, dtype=dtype)
    if kind in ("attention", "step"):
        c.update(hq=hq, causal=causal, window=window, lse=lse)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a server's step with one token for each of 64 requests: one call's latency
        _case("tables_decode", "tables", 64, 1, 4096, 0, 1, 1, 16, 1),
        # thousands of requests, some bringing prompts: 4096 table rows, up to 2^18 tokens
        _case("tables_prompts", "tables", 4096, 0, 4096, 256, 1, 1800, 16, 2, pad=64),
        # the keys and values of one step of 200 single tokens
        _case("write_decode", "write", 200, 1, 2048, 0, 1, 1, 16, 3),
        # of prompts, 24 thousand tokens in all
        _case("write_prompts", "write", 12, 0, 512, 12, 1000, 3000, 64, 4),
        # one conversation, one token: latency
        _case("decode_one", "attention", 1, 2000, 2000, 0, 1, 1, 16, 5),
        # a full batch of conversations of every length, bound by the cache's bytes
        _case("decode_batch", "attention", 128, 16, 8192, 0, 1, 1, 16, 6),
        # two long documents, four tokens checked at once, many query heads to a shared head
        _case("decode_long_f16", "attention", 2, 100001, 131000, 2, 4, 4, 32, 7, hq=64, hkv=8, dtype="f16", lse=True),
        # encoder heads of 64, 12 sequences of up to 512 tokens, no mask, no shared heads
        _case("encoder_64", "attention", 12, 0, 0, 12, 350, 512, 32, 8, hq=16, hkv=16, d=64, causal=False, lse=True),
        # a chunk of a long prompt over what is cached of it
        _case("chunk", "attention", 1, 6100, 6100, 1, 2048, 2048, 64, 9),
        # whole prompts under a sliding window, an odd number of query heads to a shared one
        _case("window", "attention", 3, 0, 1000, 3, 2000, 6000, 16, 10, hq=20, hkv=4, window=1024),
        # two whole prompts of 8192 tokens: the most work
        _case("prompts", "attention", 2, 0, 0, 2, 8192, 8192, 64, 11),
        # a mixed step as a server runs it: 47 single tokens and one chunk; tables, write, attention
        _case("step_mixed", "step", 48, 100, 3000, 1, 700, 900, 16, 12),
    ]


def _log(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    """One more case of these ranges, odd sizes among them."""
    while True:
        kind = rng.choice(["tables", "write", "attention", "attention", "attention", "step"])
        few = rng.random() < 0.4
        n = _log(rng, 1, 8) if few else _log(rng, 4, 4096 if kind == "tables" else 160)
        cached = 0 if rng.random() < 0.2 else _log(rng, 16, 130000 if n <= 4 else 9000)
        chunks = min(n, rng.choice([0, 1, 4, n if n <= 16 else 8]))
        new = _log(rng, 4, 8192)
        page = rng.choice([8, 16, 16, 32, 48, 64, 128, 256, 1])
        hkv, g = rng.choice([1, 2, 4, 8, 5]), rng.choice([1, 2, 4, 8, 3, 5, 16])
        if kind != "tables" and page == 1:
            page = 16
        c = _case(None, kind, n, min(cached, rng.choice([0, 1, cached])), cached, chunks, max(1, new // 2), new, page,
                  rng.randrange(1 << 30), hq=hkv * g, hkv=hkv, d=rng.choice([64, 128, 128, 80, 96]),
                  dtype=rng.choice(["bf16", "bf16", "f16"]), causal=True,
                  window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]), lse=rng.random() < 0.3, pad=rng.choice([1, 8, 64]))
        if kind == "attention" and rng.random() < 0.2:
            c.update(causal=False, window=0)
        if c.get("hq", 0) * c.get("d", 0) == 3072:
            continue
        cl, fl = _lens(c)
        w = work(c)
        if int(fl.sum()) > _MAX_TOKENS or w["bytes"] > _MAX_BYTES or w["flops"] > _MAX_FLOPS:
            continue
        if kind == "tables" and n * (int((cl + fl).max()) // page + 1) > 1 << 24:
            continue
        if kind != "tables" and int((cl + fl).sum()) * c["hkv"] * c["d"] > 1 << 29:
            continue
        if kind != "tables" and int((cl + fl).sum()) < 64:
            continue
        return c


def _lens(case):
    """(cached, fresh) of every request."""
    g = np.random.default_rng(case["lens_seed"])
    n = case["n"]
    cached = g.integers(case["cached_min"], case["cached"] + 1, n)
    fresh = np.ones(n, np.int64)
    who = g.permutation(n)[:case["chunks"]]
    fresh[who] = g.integers(case["new_min"], case["new"] + 1, len(who))
    return cached.astype(np.int64), fresh


def _tokens(case, fresh):
    """Tokens of the step, rounded up as a program with fixed sizes pads them."""
    return -(-int(fresh.sum()) // case["pad"]) * case["pad"]


def _normal(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(_TORCH[dtype])


def _inputs(case, seed):
    """What the program holds before the call, by name."""
    cached, fresh = _lens(case)
    kind, P, n = case["kind"], case["page"], case["n"]
    have, need = -(-cached // P), -(-(cached + fresh) // P)
    width = int(need.max()) + 3
    pages = int(need.sum()) + int(need.sum()) // 4 + 8
    order = np.random.default_rng(seed).permutation(pages).astype(np.int32)
    full = np.zeros((n, width), np.int32)
    col = np.arange(width)
    filled = np.where(kind in ("tables", "step"), have, need)
    # pages of the first `filled` entries; the rest of the pool is free
    mine = np.cumsum(filled) - filled
    sel = col[None, :] < filled[:, None]
    full[sel] = order[(mine[:, None] + col[None, :])[sel]]
    free = order[int(filled.sum()):]
    t = dict(case=case, cached_h=cached.tolist(), fresh_h=fresh.tolist(), max_new=int(fresh.max()),
             cached=torch.tensor(cached, dtype=torch.int32, device="cuda"),
             fresh=torch.tensor(fresh, dtype=torch.int32, device="cuda"),
             free=torch.from_numpy(free.copy()).cuda(), tables=torch.from_numpy(full).cuda())
    T = _tokens(case, fresh)
    starts = np.concatenate([[0], np.cumsum(fresh)])
    owner = np.repeat(np.arange(n), fresh)
    pos = cached[owner] + np.arange(len(owner)) - starts[owner]
    if kind in ("attention", "write"):
        slots = np.full(T, -1, np.int64)
        slots[:len(owner)] = full[owner, pos // P].astype(np.int64) * P + pos % P
        t.update(starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                 lengths=torch.tensor(cached + fresh, dtype=torch.int32, device="cuda"),
                 slots=torch.from_numpy(slots).cuda())
    else:
        new = lambda m, dt: torch.zeros(m, dtype=dt, device="cuda")
        t.update(starts=new(n + 1, torch.int32), lengths=new(n, torch.int32), slots=new(T, torch.int64),
                 positions=new(T, torch.int32), owners=new(T, torch.int32), info=new(4, torch.int64))
    if kind == "tables":
        return t
    dt, hkv, d = case["dtype"], case["hkv"], case["d"]
    t["kc"] = _normal((pages, P, hkv, d), 5 * seed, dt)
    t["vc"] = _normal((pages, P, hkv, d), 5 * seed + 1, dt)
    if kind in ("write", "step"):
        t["k"] = _normal((T, hkv, d), 5 * seed + 2, dt)
        t["v"] = _normal((T, hkv, d), 5 * seed + 3, dt)
    if kind in ("attention", "step"):
        t["q"] = _normal((T, case["hq"], d), 5 * seed + 4, dt, 2.0)
        t["scale"] = d ** -0.5
    return t


def prepare(case, seed):
    st = _inputs(case, seed)
    if case["kind"] in ("attention", "step"):
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(st["q"].shape[:2], device="cuda") if case["lse"] else None
        if own:
            from paper_2002_07062_gb300 import bsm
            nb = bsm.bsm_paged_workspace_bytes(case["hq"], case["hkv"], case["d"], st["max_new"])
            st["work"] = torch.zeros(nb, dtype=torch.uint8, device="cuda")
    return st


def _plain_tables(s):
    P, tab, free = s["case"]["page"], s["tables"], s["free"]
    n, width = tab.shape
    T = s["slots"].numel()
    cached, fresh = s["cached"].long(), s["fresh"].long()
    have, need = (cached + P - 1) // P, (cached + fresh + P - 1) // P
    take = need - have
    first = torch.cumsum(take, 0) - take
    ends = torch.cumsum(fresh, 0)
    begin = ends - fresh
    s["starts"][:1] = 0
    s["starts"][1:] = ends.int()
    s["lengths"][:] = (cached + fresh).int()
    col = torch.arange(width, device="cuda")
    at = first[:, None] + col - have[:, None]
    isnew = (col >= have[:, None]) & (col < need[:, None])
    page = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    tab[:] = torch.where(isnew, page, tab)
    step = torch.zeros(T + 1, dtype=torch.int64, device="cuda")
    step.index_add_(0, ends, torch.ones_like(ends))
    t = torch.arange(T, device="cuda")
    own_ = torch.cumsum(step, 0)[:T]
    live = t < ends[-1]
    own_ = torch.where(live, own_, 0)
    pos = torch.where(live, cached[own_] + t - begin[own_], 0)
    pg = tab[own_, pos // P].long()
    s["slots"][:] = torch.where(live & (pg >= 0), pg * P + pos % P, -1)
    s["positions"][:] = torch.where(live, pos, -1).int()
    s["owners"][:] = torch.where(live, own_, -1).int()
    s["info"][0] = ends[-1]
    s["info"][1] = take.sum().clamp(max=free.numel())
    s["info"][2] = (take.sum() - free.numel()).clamp(min=0)
    s["info"][3] = 0


def _plain_write(s):
    live = (s["slots"] >= 0).nonzero().view(-1)
    at = s["slots"][live]
    for cache, new in ((s["kc"], s["k"]), (s["vc"], s["v"])):
        cache.view(-1, *cache.shape[2:])[at] = new[live]


def _plain_attention(s):
    c = s["case"]
    hkv, g, d, P = c["hkv"], c["hq"] // c["hkv"], c["d"], c["page"]
    t0 = 0
    for r, (old, m) in enumerate(zip(s["cached_h"], s["fresh_h"])):
        L = old + m
        pages = s["tables"][r, :-(-L // P)].long()
        k = s["kc"][pages].view(-1, hkv, d)[:L].float().permute(1, 2, 0)
        v = s["vc"][pages].view(-1, hkv, d)[:L].float().permute(1, 0, 2)
        key = torch.arange(L, device="cuda")
        step = max(1, _ROWS // (c["hq"] * L))
        for a in range(0, m, step):
            b = min(m, a + step)
            q = s["q"][t0 + a:t0 + b].float().view(b - a, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, (b - a) * g, d)
            x = (q @ k).mul_(s["scale"])
            if c["causal"]:
                at = (old + torch.arange(a, b, device="cuda")).repeat_interleave(g)[:, None]
                hide = key > at
                if c["window"]:
                    hide = hide | (key <= at - c["window"])
                x.masked_fill_(hide, float("-inf"))
            top = x.amax(-1, keepdim=True)
            top = torch.where(top == float("-inf"), 0.0, top)
            e = x.sub_(top).exp_()
            total = e.sum(-1, keepdim=True)
            o = (e @ v) / torch.where(total > 0, total, 1.0)
            back = lambda z: z.view(hkv, b - a, g, -1).permute(1, 0, 2, 3).reshape(b - a, c["hq"], -1)
            s["out"][t0 + a:t0 + b] = back(o).to(s["out"].dtype)
            if s["lse"] is not None:
                s["lse"][t0 + a:t0 + b] = back(top + total.log())[..., 0]
        t0 += m


def _outputs(s):
    kind = s["case"]["kind"]
    out = {}
    if kind in ("tables", "step"):
        out.update({k: s[k] for k in ("tables", "starts", "lengths", "slots", "positions", "owners", "info")})
    if kind in ("write", "step"):
        out.update(kc=s["kc"], vc=s["vc"])
    if kind in ("attention", "step"):
        out["out"] = s["out"]
        if s["lse"] is not None:
            out["lse"] = s["lse"]
    return out


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        from paper_2002_07062_gb300 import bsm
        st = torch.cuda.current_stream()
        if kind in ("tables", "step"):
            bsm.bsm_paged_tables(s["cached"], s["fresh"], s["free"], s["case"]["page"], s["tables"], s["starts"],
                                 s["lengths"], s["slots"], s["positions"], s["owners"], s["info"], stream=st)
        if kind in ("write", "step"):
            bsm.bsm_paged_write(s["k"], s["v"], s["kc"], s["vc"], s["slots"], stream=st)
        if kind in ("attention", "step"):
            bsm.bsm_paged_attention(s["q"], s["kc"], s["vc"], s["out"], s["starts"], s["lengths"], s["tables"],
                                    s["max_new"], s["scale"], s["work"],
                                    flags=bsm.FLAG_CAUSAL if s["case"]["causal"] else 0, window=s["case"]["window"],
                                    lse=s["lse"], stream=st)
    else:
        if kind in ("tables", "step"):
            _plain_tables(s)
        if kind in ("write", "step"):
            _plain_write(s)
        if kind in ("attention", "step"):
            _plain_attention(s)
    return _outputs(s)


def _pairs(case, cached, fresh):
    """Visible (query, key) pairs of every request, and the keys any query sees."""
    L = cached + fresh
    if not case["causal"]:
        return fresh * L, L
    w = case["window"] or int(L.max())
    pairs = np.array([int(np.minimum(np.arange(c + 1, l + 1), w).sum()) for c, l in zip(cached, L)])
    return pairs, np.minimum(L, fresh + w - 1)


def work(case):
    """Each input read once, each output written once; two products of 2 d
    operations for every visible pair and query head."""
    cached, fresh = _lens(case)
    P, T, n = case["page"], int(fresh.sum()), case["n"]
    have, need = -(-cached // P), -(-(cached + fresh) // P)
    by = fl = 0
    if case["kind"] in ("tables", "step"):
        taken = int((need - have).sum())
        by += 8 * n + 4 * (2 * n + 1) + 16 * _tokens(case, fresh) + 8 * taken + 32
        fl += 8 * T + 4 * n
    if case["kind"] in ("write", "step"):
        by += 8 * _tokens(case, fresh) + 4 * T * case["hkv"] * case["d"] * 2
        fl += T
    if case["kind"] in ("attention", "step"):
        pairs, seen = _pairs(case, cached, fresh)
        by += int(seen.sum()) * case["hkv"] * case["d"] * 4 + 4 * T * case["hq"] * case["d"]
        by += 4 * int(need.sum()) + 4 * (2 * n + 1) + (4 * T * case["hq"] if case["lse"] else 0)
        fl += 4 * int(pairs.sum()) * case["hq"] * case["d"]
    return {"bytes": by, "flops": fl}


def exact(case, seed):
    """Attention from its definition in 64 bits, head by head and request by
    request; a write's caches hold the given values; tables are whole numbers."""
    kind = case["kind"]
    if kind == "tables":
        return None
    s = _inputs(case, seed)
    cached, fresh = _lens(case)
    P, n = case["page"], case["n"]
    kc, vc = s["kc"].double(), s["vc"].double()
    tables = s["tables"].cpu().numpy().astype(np.int64)
    res = {}
    if kind == "step":
        # new pages go out in request order
        free, nxt = s["free"].cpu().numpy(), 0
        for r in range(n):
            for j in range(-(-int(cached[r]) // P), -(-int(cached[r] + fresh[r]) // P)):
                tables[r, j] = free[nxt]
                nxt += 1
        res.update({k: None for k in ("tables", "starts", "lengths", "slots", "positions", "owners", "info")})
    rows = [torch.from_numpy(tables[r, np.arange(int(cached[r] + fresh[r])) // P] * P
                             + np.arange(int(cached[r] + fresh[r])) % P).cuda() for r in range(n)]
    if kind in ("write", "step"):
        t0 = 0
        for r in range(n):
            m, old = int(fresh[r]), int(cached[r])
            for cache, new in ((kc, s["k"]), (vc, s["v"])):
                cache.view(-1, case["hkv"], case["d"])[rows[r][old:]] = new[t0:t0 + m].double()
            t0 += m
        res.update(kc=kc, vc=vc)
        if kind == "write":
            return res
    T, hq, d, g = s["q"].shape[0], case["hq"], case["d"], case["hq"] // case["hkv"]
    out = torch.zeros((T, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((T, hq), dtype=torch.float64, device="cuda")
    t0 = 0
    for r in range(n):
        m, old = int(fresh[r]), int(cached[r])
        keys = torch.arange(old + m, device="cuda")
        for h in range(case["hkv"]):
            kd = kc.view(-1, case["hkv"], d)[rows[r], h]
            vd = vc.view(-1, case["hkv"], d)[rows[r], h]
            for i in range(0, m, max(1, (1 << 25) // (g * (old + m)))):
                j = min(m, i + max(1, (1 << 25) // (g * (old + m))))
                z = torch.einsum("ihd,kd->ihk", s["q"][t0 + i:t0 + j, h * g:(h + 1) * g].double(), kd) * s["scale"]
                if case["causal"]:
                    far = old + torch.arange(i, j, device="cuda")[:, None] - keys[None, :]
                    ok = far >= 0
                    if case["window"]:
                        ok &= far < case["window"]
                    z = torch.where(ok[:, None, :], z, torch.full_like(z, float("-inf")))
                ls = torch.logsumexp(z, -1)
                out[t0 + i:t0 + j, h * g:(h + 1) * g] = torch.einsum("ihk,kd->ihd", torch.exp(z - ls[..., None]), vd)
                lse[t0 + i:t0 + j, h * g:(h + 1) * g] = ls
        t0 += m
    res["out"] = out
    if case["lse"]:
        res["lse"] = lse
    return res
