"""Decode steps with beams over the paged cache, all calls together: tables, rotary
write, attention, selection, reordering in place; every step against histories kept
on the host."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import beam_oracle as O
from oracle import paged_oracle as OP
from paper_2002_07062_gb300 import bsm

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n,B,page,hq,hkv,d,rot,inter,prompt,steps,dtype", [
    (3, 4, 16, 8, 2, 64, 64, False, (5, 40), 9, torch.bfloat16),
    (2, 5, 8, 6, 3, 128, 32, True, (1, 20), 12, torch.float16),
    (5, 2, 16, 4, 4, 64, 64, True, (15, 17), 6, torch.bfloat16),
])
def test_steps_follow_the_histories(n, B, page, hq, hkv, d, rot, inter, prompt, steps, dtype):
    rng = np.random.default_rng(n * 100 + B)
    V, layers, rows, end = 300, 2, n * B, 7
    g = torch.Generator(device="cuda").manual_seed(n)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    # queries, keys and values of a token in a layer; logits from the last layer's output
    tok = [rnd(V, hq + 2 * hkv, d).to(dtype) for _ in range(layers)]
    head = rnd(hq * d, V) * 0.4
    lens = rng.integers(prompt[0], prompt[1] + 1, n)
    width = -(-int(lens.max() + steps + 1) // page)
    pages = rows * width + 5
    kc, vc = (torch.full((layers, pages, page, hkv, d), float("nan"), device="cuda").to(dtype) for _ in range(2))
    most = int(lens.max()) + steps + 2
    angle = torch.arange(most, dtype=torch.float64, device="cuda")[:, None] * \
        10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    table = torch.cat([angle.cos(), angle.sin()], 1).float()
    free = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    tables, cached = torch.full((rows, width), -1, dtype=torch.int32, device="cuda"), _i32([0] * rows)
    starts, lengths = _i32([0] * (rows + 1)), _i32([0] * rows)
    dropped, info = _i32([0] * (rows * width)), torch.zeros(4, dtype=torch.int64, device="cuda")
    ws = torch.empty(bsm.bsm_paged_workspace_bytes(hq, hkv, d, int(lens.max())), dtype=torch.uint8, device="cuda")
    ws_s = torch.empty(bsm.bsm_beam_select_workspace_bytes(n, B, V, B), dtype=torch.uint8, device="cuda")
    ws_r = torch.empty(bsm.bsm_paged_reorder_workspace_bytes(n, B, width), dtype=torch.uint8, device="cuda")
    hist = [rng.integers(0, V, lens[r // B]).tolist() if r % B == 0 else None for r in range(rows)]
    new = [h or [] for h in hist]                       # tokens that go into the cache in this step
    scores = torch.full((n, B), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    ended = torch.zeros((n, B), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        fresh, T = _i32([len(x) for x in new]), sum(len(x) for x in new)
        pad = T + 3
        slots = torch.empty(pad, dtype=torch.int64, device="cuda")
        pos, own = torch.empty((2, pad), dtype=torch.int32, device="cuda")
        bsm.bsm_paged_tables(cached, fresh, free, page, tables, starts, lengths, slots, pos, own, info)
        taken, missing, flags = info.tolist()[1:]
        assert missing == 0 and flags == 0
        free = free[taken:]
        ids = torch.tensor([t for x in new for t in x] + [0, 0, 0], device="cuda")
        for layer in range(layers):
            qkv = tok[layer][ids]
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            bsm.bsm_paged_write_rotary(q, k, v, q, kc[layer], vc[layer], slots, pos, table,
                                       flags=bsm.FLAG_INTERLEAVED if inter else 0)
            out = torch.zeros_like(q)
            bsm.bsm_paged_attention(q, kc[layer], vc[layer], out, starts, lengths, tables, max(len(x) for x in new), d ** -0.5,
                                    ws, flags=bsm.FLAG_CAUSAL)
        last = (starts[1:].long() - 1).clamp(min=0)
        logits = (out[last].float().view(rows, hq * d) @ head).to(dtype).view(n, B, V)
        new_scores, parents, tokens = torch.empty((n, B), device="cuda"), *torch.empty((2, n, B), dtype=torch.int32, device="cuda")
        bsm.bsm_beam_select(logits, scores, new_scores, parents, tokens, ws_s, ended=ended, end_token=end)
        # the histories: keys and values where the tables say, and attention over them
        tab = tables.tolist()
        for r in range(rows):
            if hist[r] is None or not new[r]:
                continue
            L = len(hist[r])
            assert int(lengths[r]) == L
            t = torch.tensor(hist[r], device="cuda")
            place = torch.tensor([tab[r][p // page] * page + p % page for p in range(L)], device="cuda")
            for layer in range(layers):
                ref, size = O.rotary(tok[layer][t][:, hq:hq + hkv], range(L), table, inter)
                got = kc[layer].view(-1, hkv, d)[place].double()
                assert ((got - ref).abs() <= torch.finfo(dtype).eps / 2 * ref.abs() * 1.001 + 2.0 ** -21 * size + 1e-6).all()
                assert torch.equal(vc[layer].view(-1, hkv, d)[place], tok[layer][t][:, hq + hkv:])
        ref, _, mass, size = OP.attention(q[:T], kc[layers - 1], vc[layers - 1], starts.tolist(), lengths.tolist(), tab, d ** -0.5, True)
        # probabilities rounded to the type, the output once more (and fp32 sums over a few hundred terms)
        err = (out[:T].double() - ref).abs()
        assert (err <= torch.finfo(dtype).eps * (2 * mass + ref.abs()) + 1e-4).all(), float(err.max())
        val, par, tk = O.select(logits.double().cpu().numpy(), scores.cpu().numpy(), B, ended.cpu().numpy(), end)
        assert np.abs(np.where(np.isfinite(val), new_scores.cpu().numpy() - np.where(np.isfinite(val), val, 0), 0)).max() < 1e-4
        same = (parents.cpu().numpy() == par) & (tokens.cpu().numpy() == tk)
        assert same.mean() > 0.9                        # (near-equal candidates may trade places)
        # the cache follows, in place
        before = tables.clone()
        bsm.bsm_paged_reorder(parents, lengths, tables, free, lengths, tables, dropped, info, kc, vc, ws_r)
        taken, missing, gone, flags = info.tolist()
        assert missing == 0 and flags == 0
        free = torch.cat([free[taken:], dropped[:gone]])
        cached = lengths.clone()
        p, t = parents.view(-1).tolist(), tokens.view(-1).tolist()
        was_ended = ended.view(-1).tolist()
        old = hist
        hist, new, end_flags = [], [], []
        for r in range(rows):
            src = r // B * B + p[r]
            if p[r] < 0:
                hist.append(None)
                new.append([])
                end_flags.append(0)
            elif was_ended[src]:
                hist.append(old[src])
                new.append([])
                end_flags.append(1)
            else:
                hist.append(old[src] + [t[r]])
                new.append([t[r]])
                end_flags.append(int(t[r] == end))
        scores, ended = new_scores, torch.tensor(end_flags, dtype=torch.uint8, device="cuda").view(n, B)
        # no page is lost, and none is free and held
        held = set()
        tab = tables.tolist()
        for r in range(rows):
            held |= set(tab[r][:-(-int(lengths[r]) // page)])
        assert sorted(list(held) + free.tolist()) == list(range(pages))
        assert not torch.equal(before, tables) or step > 0 or B == 1
    assert bsm.bsm_device_status() == 0


def test_example_runs():
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_search.py")
    spec = importlib.util.spec_from_file_location("beam_search", at)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    # bf16 keys and probabilities against float64: a few roundings of 2^-8
    assert m.main(["--requests", "3", "--beams", "4", "--steps", "10", "--layers", "2", "--vocab", "1000", "--check"]) < 0.05


@pytest.mark.parametrize("steps", [1, 2])
def test_example_checks_its_first_steps(steps):
    # in the first one only one beam of a request has a history
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_search.py")
    spec = importlib.util.spec_from_file_location("beam_search_first", at)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    worst = m.main(["--requests", "2", "--beams", "3", "--steps", str(steps), "--layers", "2", "--vocab", "500", "--prompt", "40",
                    "--check"])
    assert 0.0 < worst < 0.05


def test_example_has_pages_for_copies_that_come_before_dropped_ones():
    # a page a row holds everything; a step whose rows share a beam takes one more
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_search.py")
    spec = importlib.util.spec_from_file_location("beam_search_small", at)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main(["--requests", "1", "--beams", "4", "--steps", "15", "--layers", "1", "--vocab", "300", "--prompt", "1",
                   "--check"]) < 0.05
