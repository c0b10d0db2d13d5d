"""The operators of a decode step with beams over the paged cache, as they are
measured: new keys and values rotated by their positions on the way to their
slots (queries too), the selection of continuations over beams and vocabulary,
and the cache's tables and partly filled pages following the selected beams.

A case is a dict:
  kind    "append", "select" or "reorder"
  append  n requests with cached_min..cached tokens, each bringing new_min..new
          more; tokens rounded up to a multiple of `pad`; hq, hkv, d heads and
          their size, rot the rotated columns, inter pairs side by side, page
          tokens a page holds
  select  n requests of `beams` rows of `vocab` logits (`gap` more columns from
          row to row), `keep` continuations; `ended` the share of finished beams,
          dead: only the first beam of each request has a score yet; masked: the
          share of logits at -inf
  reorder n requests of `beams` rows of lo..hi tokens, `prompt` of them shared;
          spread: how evenly the beams are chosen (0: one beam's children all);
          layers, hkv, d, page of the caches
  dtype   "bf16", "f16", "f32";  case_seed draws lengths and parents
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
_MAX_BYTES = 700_000_000        # a drawn case's at most; the largest listed ones' are a little more


def _append(name, n, cached_min, cached, new_min, new, page, case_seed, hq=32, hkv=8, d=128, rot=128, inter=False,
            dtype="bf16", pad=1):
    c = dict(kind="append", n=n, cached_min=cached_min, cached=cached, new_min=new_min, new=new, page=page, hq=hq, hkv=hkv,
             d=d, rot=rot, inter=inter, dtype=dtype, pad=pad, case_seed=case_seed)
    return dict(c, name=name) if name else c


def _select(name, n, beams, vocab, keep, dtype="bf16", gap=0, ended=0.0, dead=False, masked=0.0, case_seed=0):
    c = dict(kind="select", n=n, beams=beams, vocab=vocab, keep=keep, dtype=dtype, gap=gap, ended=ended, dead=dead,
             masked=masked, case_seed=case_seed)
    return dict(c, name=name) if name else c


def _reorder(name, n, beams, prompt, lo, hi, page, layers, case_seed, spread=1.0, hkv=8, d=128, dtype="bf16"):
    c = dict(kind="reorder", n=n, beams=beams, prompt=prompt, lo=lo, hi=hi, page=page, layers=layers, spread=spread,
             hkv=hkv, d=d, dtype=dtype, case_seed=case_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one conversation's token in one layer: the latency of a call
        _append("append_one", 1, 4000, 4000, 1, 1, 16, 1),
        # a server's step: a token for each of 256 rows
        _append("append_decode", 256, 1, 8000, 1, 1, 16, 2),
        # prompts in chunks, a third of a head rotated with its pairs side by side, an odd number of heads
        _append("append_partial_f16", 5, 0, 30000, 100, 900, 48, 3, hq=15, hkv=5, d=96, rot=32, inter=True, dtype="f16", pad=8),
        # whole prompts, 40 thousand tokens: the largest write
        _append("append_prompts", 16, 0, 0, 1000, 4000, 64, 4, pad=64),
        # one request's four beams: latency
        _select("select_one", 1, 4, 32000, 8),
        # the first step after a prompt: one live beam of five, rows that start at odd addresses
        _select("select_first", 24, 5, 50001, 10, ended=0.0, dead=True),
        # fp32 logits, some beams finished, most of the vocabulary forbidden by a grammar in a padded row
        _select("select_masked_f32", 32, 8, 100000, 16, dtype="f32", gap=64, ended=0.2, masked=0.9, case_seed=7),
        # a full server: 128 requests of 8 beams over a large vocabulary, the largest selection
        _select("select_full", 128, 8, 128000, 16, ended=0.05, case_seed=8),
        # one request's four beams in one layer: latency
        _reorder("reorder_one", 1, 4, 300, 310, 340, 16, 1, 9),
        # a server's 64 requests of 5 beams in small pages, every layer
        _reorder("reorder_small_pages", 64, 5, 200, 201, 700, 16, 24, 10, d=64),
        # large pages: the copies are the work
        _reorder("reorder_large_pages", 32, 8, 100, 130, 400, 64, 16, 11),
        # tables of long histories, one layer, many rows
        _reorder("reorder_long", 16, 16, 16000, 17000, 24000, 16, 1, 12, spread=0.5, hkv=2, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    """One more case of these ranges, odd sizes among them."""
    while True:
        kind = rng.choice(["append", "select", "reorder"])
        seed = rng.randrange(1 << 30)
        if kind == "append":
            d = rng.choice([64, 128, 128, 80, 96, 256])
            hkv = rng.choice([1, 2, 4, 8, 5])
            long_ = rng.random() < 0.5
            cached = 0 if rng.random() < 0.2 else _log(rng, 16, 100000)
            new = _log(rng, 2, 4000) if long_ else 1
            c = _append(None, _log(rng, 1, 16 if long_ else 512), min(cached, rng.choice([0, cached])), cached,
                        max(1, new // 3), new, rng.choice([16, 16, 32, 64, 48, 1, 100]), seed,
                        hq=hkv * rng.choice([1, 2, 3, 4, 8]), hkv=hkv, d=d, rot=rng.choice([d, d, d, d // 2, 32, 20]),
                        inter=rng.random() < 0.4, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                        pad=rng.choice([1, 8, 64]))
        elif kind == "select":
            beams = rng.choice([1, 2, 4, 4, 5, 8, 16, 3])
            c = _select(None, _log(rng, 1, 128), beams, _log(rng, 500, 260000), min(64, beams * rng.choice([1, 2, 2, 3])),
                        dtype=rng.choice(["bf16", "bf16", "f32", "f16"]), gap=rng.choice([0, 0, 1, 64]),
                        ended=rng.choice([0.0, 0.1, 0.5]), dead=rng.random() < 0.15, masked=rng.choice([0.0, 0.0, 0.5, 0.99]),
                        case_seed=seed)
        else:
            lo = _log(rng, 2, 20000)
            c = _reorder(None, _log(rng, 1, 128), rng.choice([2, 4, 4, 5, 8, 16, 3]), rng.randrange(0, lo), lo,
                         lo + _log(rng, 1, 1000), rng.choice([16, 16, 32, 64, 8, 100]), _log(rng, 1, 32), seed,
                         spread=rng.choice([1.0, 0.5, 0.0]), hkv=rng.choice([1, 2, 4, 8, 5]), d=rng.choice([64, 128, 96]),
                         dtype=rng.choice(["bf16", "bf16", "f16"]))
            if _pool(c) * c["page"] * c["hkv"] * c["d"] * c["layers"] > 1 << 31:
                continue
        if work(c)["bytes"] <= _MAX_BYTES:
            return c


def _normal(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(_TORCH[dtype])


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- what a program has in hand ----

def _tokens(c):
    """(tokens with their padding, positions and owners of the real ones, cached, fresh)."""
    g = np.random.default_rng(c["case_seed"])
    cached = g.integers(c["cached_min"], c["cached"] + 1, c["n"])
    fresh = g.integers(c["new_min"], c["new"] + 1, c["n"])
    owner = np.repeat(np.arange(c["n"]), fresh)
    at = np.arange(len(owner)) - (np.cumsum(fresh) - fresh)[owner]
    return -(-len(owner) // c["pad"]) * c["pad"], cached[owner] + at, owner, cached, fresh


def _append_state(c, seed):
    T, pos, owner, cached, fresh = _tokens(c)
    P, m = c["page"], len(owner)
    # pages that the new tokens touch; the pool holds some more
    first, last = cached // P, (cached + fresh - 1) // P
    base = np.cumsum(last - first + 1) - (last - first + 1)
    pages = int((last - first + 1).sum()) * 5 // 4 + 8
    order = np.random.default_rng(seed).permutation(pages)
    slots, positions = np.full(T, -1, np.int64), np.full(T, -1, np.int32)
    slots[:m] = order[base[owner] + pos // P - first[owner]] * P + pos % P
    positions[:m] = pos
    most = int((cached + fresh).max())
    inv = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
    angle = torch.arange(most, dtype=torch.float64, device="cuda")[:, None] * inv
    hq, hkv = c["hq"], c["hkv"]
    qkv = _normal((T, hq + 2 * hkv, c["d"]), 3 * seed, c["dtype"])      # one projection's output
    return dict(case=c, q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:],
                q_out=torch.zeros((T, hq, c["d"]), dtype=qkv.dtype, device="cuda"),
                kc=_normal((pages, P, hkv, c["d"]), 3 * seed + 1, c["dtype"]),
                vc=_normal((pages, P, hkv, c["d"]), 3 * seed + 2, c["dtype"]),
                slots=_dev(slots), positions=_dev(positions),
                table=torch.cat([angle.cos(), angle.sin()], 1).float())


def _ended(c):
    return np.random.default_rng(c["case_seed"]).uniform(size=(c["n"], c["beams"])) < c["ended"]


def _select_state(c, seed):
    n, B, V = c["n"], c["beams"], c["vocab"]
    g = np.random.default_rng(seed)
    full = torch.empty((n, B, V + c["gap"]), dtype=_TORCH[c["dtype"]], device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(7 * seed + 1)
    for r in range(n):              # (request by request: fp32 temporaries stay small)
        x = torch.randn((B, V + c["gap"]), generator=gen, device="cuda").mul_(2.5)
        if c["masked"]:
            allowed = torch.rand((B, V + c["gap"]), generator=gen, device="cuda") >= c["masked"]
            x = torch.where(allowed, x, float("-inf"))
        full[r] = x.to(full.dtype)
    scores = -g.uniform(0.0, 30.0, (n, 1)) - np.cumsum(g.exponential(0.7, (n, B)), 1)
    if c["dead"]:
        scores[:, 1:] = -np.inf
    ended = _ended(c).astype(np.uint8) if c["ended"] else None
    K = c["keep"]
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(case=c, logits=full[:, :, :V], scores=_dev(scores.astype(np.float32)),
                ended=None if ended is None else _dev(ended), end_token=2 % V,
                out_scores=torch.zeros((n, K), device="cuda"), parents=torch.zeros((n, K), **i32),
                tokens=torch.zeros((n, K), **i32))


def _rows(c):
    """(lengths [n, beams], parents [n, beams]) of a reorder case."""
    g = np.random.default_rng(c["case_seed"])
    n, B = c["n"], c["beams"]
    lengths = np.repeat(g.integers(c["lo"], c["hi"] + 1, (n, 1)), B, 1)
    ended = g.uniform(size=(n, B)) < 0.1            # finished beams stopped growing
    lengths = np.where(ended, np.maximum(lengths - g.integers(0, 20, (n, B)), c["prompt"]), lengths)
    weight = np.exp(-np.arange(B) * 4.0 * (1.0 - c["spread"]))
    parents = np.stack([g.choice(B, B, p=weight / weight.sum()) for _ in range(n)])
    return lengths, parents


def _pool(c):
    lengths, _ = _rows(c)
    own_ = -(-lengths // c["page"]) - c["prompt"] // c["page"]
    return int(own_.sum()) + c["n"] * (c["prompt"] // c["page"]) + c["n"] * c["beams"] + 8


def _reorder_state(c, seed):
    n, B, P = c["n"], c["beams"], c["page"]
    lengths, parents = _rows(c)
    shared, need = c["prompt"] // P, -(-lengths // P)
    width = int(need.max()) + 3
    pages = _pool(c)
    order = np.random.default_rng(seed).permutation(pages).astype(np.int32)
    tables = np.full((n, B, width), -1, np.int32)
    tables[:, :, :shared] = order[:n * shared].reshape(n, 1, shared)
    col = np.arange(width)
    mine = (col >= shared) & (col < need[:, :, None])
    tables[mine] = order[n * shared:n * shared + int(mine.sum())]
    free = order[n * shared + int(mine.sum()):]
    shape = (c["layers"], pages, P, c["hkv"], c["d"])
    st = dict(case=c, lengths=_dev(lengths.reshape(-1).astype(np.int32)), parents=_dev(parents.astype(np.int32)),
              tables=_dev(tables.reshape(n * B, width)), free=_dev(free),
              kc=_normal(shape, 2 * seed, c["dtype"]), vc=_normal(shape, 2 * seed + 1, c["dtype"]))
    st.update(new_lengths=torch.zeros_like(st["lengths"]), new_tables=torch.full_like(st["tables"], -1),
              dropped=torch.full((n * B * width,), -1, dtype=torch.int32, device="cuda"),
              info=torch.zeros(4, dtype=torch.int64, device="cuda"))
    return st


_STATE = {"append": _append_state, "select": _select_state, "reorder": _reorder_state}


def prepare(case, seed):
    st = _STATE[case["kind"]](case, seed)
    if own and case["kind"] != "append":
        from paper_2002_07062_gb300 import bsm
        if case["kind"] == "select":
            nb = bsm.bsm_beam_select_workspace_bytes(case["n"], case["beams"], case["vocab"], case["keep"])
        else:
            nb = bsm.bsm_paged_reorder_workspace_bytes(case["n"], case["beams"], st["tables"].shape[1])
        st["work"] = torch.zeros(nb, dtype=torch.uint8, device="cuda")
    return st


# ---- plain forms ----

def _turn(x, cos, sin, rot, inter):
    """x [tokens, heads, d] fp32, its first rot columns rotated."""
    h = rot // 2
    c, s = cos[:, None, :], sin[:, None, :]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :h], x[..., h:rot])
    ra, rb = a * c - b * s, b * c + a * s
    turned = torch.stack([ra, rb], -1).flatten(-2) if inter else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(s):
    c = s["case"]
    live = (s["positions"] >= 0).nonzero().view(-1)
    row = s["table"][s["positions"][live].long()]
    cos, sin = row[:, :c["rot"] // 2], row[:, c["rot"] // 2:]
    turn = lambda x: _turn(x[live].float(), cos, sin, c["rot"], c["inter"]).to(x.dtype)
    s["q_out"][live] = turn(s["q"])
    at = s["slots"][live]
    s["kc"].view(-1, c["hkv"], c["d"])[at] = turn(s["k"])
    s["vc"].view(-1, c["hkv"], c["d"])[at] = s["v"][live]


def _plain_select(s):
    # in 64 bits: two beams' candidates may lie close together
    x = s["logits"].double()
    n, B, V = x.shape
    top = x.amax(-1, keepdim=True)
    rest = x.sub_(top)
    cand = rest - rest.exp().sum(-1, keepdim=True).log() + s["scores"].double()[..., None]
    cand = torch.where(torch.isnan(cand), float("-inf"), cand)
    if s["ended"] is not None:
        done = s["ended"].bool()
        cand = torch.where(done[..., None], float("-inf"), cand)
        cand[..., s["end_token"]] = torch.where(done, s["scores"].double(), cand[..., s["end_token"]])
    cand = cand.view(n, B * V)
    rows = torch.arange(n, device="cuda")
    for i in range(s["case"]["keep"]):
        at = cand.argmax(-1)
        best = cand[rows, at]
        there = best > float("-inf")
        s["out_scores"][:, i] = best.float()
        s["parents"][:, i] = torch.where(there, at // V, -1).int()
        s["tokens"][:, i] = torch.where(there, at % V, -1).int()
        cand[rows, at] = float("-inf")


def _plain_reorder(s):
    n, B = s["parents"].shape
    P, tab, free = s["case"]["page"], s["tables"], s["free"]
    width = tab.shape[1]
    alive = s["parents"] >= 0
    row = (torch.arange(n, device="cuda")[:, None] * B + s["parents"].clamp(min=0)).view(-1)
    alive = alive.view(-1)
    length = torch.where(alive, s["lengths"][row], 0)
    col = torch.arange(width, device="cuda")
    used = col < ((length + P - 1) // P)[:, None]
    moved = torch.where(used, tab[row], -1)
    # a partly filled page goes to the first row that takes it, later ones get a copy
    full, part = length // P, length % P
    tail = torch.where(part > 0, moved.gather(1, full.clamp(max=width - 1).long()[:, None])[:, 0], -1).view(n, B)
    same = (tail[:, :, None] == tail[:, None, :]).tril(-1).any(2) & (tail >= 0)
    again = same.view(-1).nonzero().view(-1)
    m = min(len(again), free.numel())
    page = torch.full_like(again, -1, dtype=torch.int32)
    page[:m] = free[:m]
    src = tail.view(-1)[again]
    moved[again, full[again].long()] = page
    s["new_tables"].copy_(torch.where(used, moved, s["new_tables"]))
    s["new_lengths"].copy_(length)
    # pages of the old rows that no new row of the request holds in that place, each once
    had = col < ((s["lengths"] + P - 1) // P)[:, None]
    old = torch.where(had, tab, -1).view(n, B, width)
    new = torch.where(used, moved, -1).view(n, B, width)
    gone = old >= 0
    for b in range(B):
        gone[:, b] &= ~(new == old[:, b:b + 1]).any(1)
        if b:
            gone[:, b] &= ~(old[:, :b] == old[:, b:b + 1]).any(1)
    out = old.transpose(1, 2)[gone.transpose(1, 2)]
    s["dropped"][:out.numel()] = out
    s["info"][0], s["info"][1], s["info"][2], s["info"][3] = m, len(again) - m, out.numel(), 0
    # the tokens of the partly filled pages
    page, src = page[:m].long(), src[:m].long()
    who, t = (torch.arange(P, device="cuda") < part[again[:m]][:, None]).nonzero().unbind(1)
    for cache in (s["kc"], s["vc"]):
        cache[:, page[who], t] = cache[:, src[who], t]


def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "append":
        return {k: s[k] for k in ("q_out", "kc", "vc")}
    if kind == "select":
        return {k: s[k] for k in ("out_scores", "parents", "tokens")}
    return {k: s[k] for k in ("new_lengths", "new_tables", "dropped", "info", "kc", "vc")}


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        from paper_2002_07062_gb300 import bsm
        st = torch.cuda.current_stream()
        if kind == "append":
            bsm.bsm_paged_write_rotary(s["q"], s["k"], s["v"], s["q_out"], s["kc"], s["vc"], s["slots"], s["positions"],
                                       s["table"], flags=bsm.FLAG_INTERLEAVED if s["case"]["inter"] else 0, stream=st)
        elif kind == "select":
            bsm.bsm_beam_select(s["logits"], s["scores"], s["out_scores"], s["parents"], s["tokens"], s["work"],
                                ended=s["ended"], end_token=s["end_token"], stream=st)
        else:
            bsm.bsm_paged_reorder(s["parents"], s["lengths"], s["tables"], s["free"], s["new_lengths"], s["new_tables"],
                                  s["dropped"], s["info"], s["kc"], s["vc"], s["work"], stream=st)
    else:
        {"append": _plain_append, "select": _plain_select, "reorder": _plain_reorder}[kind](s)
    return _outputs(s)


def _copies(c):
    """Rows of a reorder case whose partly filled page was taken by an earlier row."""
    lengths, parents = _rows(c)
    L = np.take_along_axis(lengths, parents, 1)
    part = L % c["page"]
    earlier = np.array([[p in row[:i] for i, p in enumerate(row)] for row in parents.tolist()])
    return lengths, L, np.where(earlier, part, 0)


def work(case):
    """Each input read once, each output written once."""
    c = case
    if c["kind"] == "append":
        T, pos, _, _, _ = _tokens(c)
        es, m = _SIZE[c["dtype"]], len(pos)
        rows = 2 * m * (c["hq"] + 2 * c["hkv"]) * c["d"] * es
        return {"bytes": rows + 12 * T + 4 * c["rot"] * len(np.unique(pos)),
                "flops": 3 * m * (c["hq"] + c["hkv"]) * c["rot"]}
    if c["kind"] == "select":
        # rows of finished and of dead beams need not be read
        x = int((~_ended(c))[:, :1 if c["dead"] else None].sum()) * c["vocab"]
        return {"bytes": x * _SIZE[c["dtype"]] + c["n"] * (5 * c["beams"] + 12 * c["keep"]), "flops": 4 * x}
    lengths, L, part = _copies(c)
    P = c["page"]
    entries = int((-(-lengths // P)).sum()) + int((-(-L // P)).sum())
    row = c["hkv"] * c["d"] * _SIZE[c["dtype"]]
    return {"bytes": 4 * entries + 12 * L.size + 32 + 4 * c["layers"] * row * int(part.sum()), "flops": entries}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    c = case
    s = _STATE[c["kind"]](c, seed)
    if c["kind"] == "append":
        _, pos, _, _, _ = _tokens(c)
        m, rot = len(pos), c["rot"]
        i = np.arange(rot // 2)
        first, second = (2 * i, 2 * i + 1) if c["inter"] else (i, i + rot // 2)
        row = s["table"].double()[torch.from_numpy(pos).cuda()]
        z = torch.complex(row[:, None, :rot // 2], row[:, None, rot // 2:])
        res = dict(q_out=s["q_out"].double(), kc=s["kc"].double(), vc=s["vc"].double())
        slot = s["slots"][:m]
        for name, to, at in (("q", res["q_out"], torch.arange(m, device="cuda")),
                             ("k", res["kc"].view(-1, c["hkv"], c["d"]), slot)):
            x = s[name][:m].double()
            w = torch.complex(x[..., first], x[..., second]) * z
            x[..., first], x[..., second] = w.real, w.imag
            to[at] = x
        res["vc"].view(-1, c["hkv"], c["d"])[slot] = s["v"][:m].double()
        return res
    if c["kind"] == "select":
        out = torch.empty((c["n"], c["keep"]), dtype=torch.float64, device="cuda")
        for r in range(c["n"]):
            parts = []
            for b in range(c["beams"]):
                score = s["scores"][r, b].double()
                if s["ended"] is not None and s["ended"][r, b]:
                    parts.append(score[None])
                    continue
                logp = torch.log_softmax(s["logits"][r, b].double(), 0)
                parts.append(score + torch.topk(logp, min(c["keep"], c["vocab"])).values)
            v = torch.cat(parts)
            v = torch.where(torch.isnan(v), float("-inf"), v).sort(descending=True).values[:c["keep"]]
            out[r] = float("-inf")
            out[r, :len(v)] = v
        return dict(out_scores=out, parents=None, tokens=None)
    # the caches hold given values, bit for bit: each copied page's tokens, row by row
    kc, vc = s["kc"].clone(), s["vc"].clone()
    lengths, L, part = _copies(c)
    _, parents = _rows(c)
    B, P, nxt = c["beams"], c["page"], 0
    tables, free = s["tables"].cpu().numpy(), s["free"].cpu().numpy()
    for r in range(c["n"]):
        for i in range(B):
            if part[r, i]:
                src = int(tables[r * B + parents[r, i], L[r, i] // P])
                kc[:, int(free[nxt]), :part[r, i]] = s["kc"][:, src, :part[r, i]]
                vc[:, int(free[nxt]), :part[r, i]] = s["vc"][:, src, :part[r, i]]
                nxt += 1
    return dict(new_lengths=None, new_tables=None, dropped=None, info=None, kc=kc, vc=vc)
