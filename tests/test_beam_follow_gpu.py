"""Many steps with beams, every entry of every call checked: the selection by the gap
between its candidates, tables, lengths, dropped pages and caches of a reordering in
place against plain loops."""
import numpy as np
import pytest
import torch

import test_beam_select_gpu as S
from oracle import beam_oracle as O
from paper_2002_07062_gb300 import bsm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,B,page,steps,dtype", [
    (6, 8, 4, 14, torch.bfloat16), (20, 3, 1, 8, torch.float16), (2, 20, 16, 20, torch.float32), (9, 2, 64, 9, torch.bfloat16)])
def test_every_step_by_its_definition(n, B, page, steps, dtype):
    bsm.bsm_device_status_clear()
    rng = np.random.default_rng(n + B)
    g = torch.Generator(device="cuda").manual_seed(n)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    V, layers, hkv, d, rot, rows, end = 400, 3, 2, 32, 16, n * B, 5
    lens = rng.integers(1, 40, n)
    width = -(-(int(lens.max()) + steps + 1) // page)
    pages = rows * width + rows         # (a copied page is taken before the dropped ones come back)
    kc, vc = (torch.full((layers, pages, page, hkv, d), 9.0, device="cuda").to(dtype) for _ in range(2))
    tok = rnd(layers, V, 2 * hkv, d).to(dtype)
    angle = torch.arange(int(lens.max()) + steps + 1, dtype=torch.float64, device="cuda")[:, None] * \
        10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    table = torch.cat([angle.cos(), angle.sin()], 1).float()
    free = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    tables, cached = torch.full((rows, width), -1, **i32), torch.zeros(rows, **i32)
    starts, lengths = torch.zeros(rows + 1, **i32), torch.zeros(rows, **i32)
    dropped, info = torch.zeros(rows * width, **i32), torch.zeros(4, dtype=torch.int64, device="cuda")
    ws_s = torch.empty(bsm.bsm_beam_select_workspace_bytes(n, B, V, B), dtype=torch.uint8, device="cuda")
    ws_r = torch.empty(bsm.bsm_paged_reorder_workspace_bytes(n, B, width), dtype=torch.uint8, device="cuda")
    new = [rng.integers(0, V, lens[r // B]).tolist() if r % B == 0 else [] for r in range(rows)]
    hist = [list(x) for x in new]
    scores = torch.full((n, B), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    ended = torch.zeros((n, B), dtype=torch.uint8, device="cuda")
    copied = gone_all = 0
    for step in range(steps):
        fresh, T = torch.tensor([len(x) for x in new], **i32), sum(len(x) for x in new)
        slots = torch.empty(max(T, 1), dtype=torch.int64, device="cuda")
        pos, own = torch.empty((2, max(T, 1)), **i32)
        bsm.bsm_paged_tables(cached, fresh, free, page, tables, starts, lengths, slots, pos, own, info)
        taken, missing, flags = info.tolist()[1:]
        assert missing == 0 and flags == 0
        free = free[taken:]
        ids = torch.tensor([t for x in new for t in x], dtype=torch.int64, device="cuda")
        for layer in range(layers if T else 0):
            kv = tok[layer][ids]
            bsm.bsm_paged_write_rotary(None, kv[:, :hkv], kv[:, hkv:], None, kc[layer], vc[layer], slots[:T], pos[:T], table)
        logits = (rnd(n, B, V) * 2).to(dtype)
        out = [torch.empty((n, B), device="cuda"), torch.empty((n, B), **i32), torch.empty((n, B), **i32)]
        bsm.bsm_beam_select(logits, scores, *out, ws_s, ended=ended, end_token=end)
        S._check(logits, scores, B, ended, end, got=out)
        new_scores, parents, tokens = out
        # the reordering in place, entry by entry
        L0, T0, F0, k0, v0 = lengths.tolist(), tables.tolist(), free.tolist(), kc.clone(), vc.clone()
        want_len, want_tab, copies, missing, want_gone = O.reorder(parents.tolist(), L0, T0, F0, page)
        bsm.bsm_paged_reorder(parents, lengths, tables, free, lengths, tables, dropped, info, kc, vc, ws_r)
        taken, _, gone, flags = info.tolist()
        assert missing == 0 and flags == 0 and taken == len(copies) and gone == len(want_gone)
        assert lengths.tolist() == want_len and dropped[:gone].tolist() == want_gone
        for (i, c), e in want_tab.items():
            T0[i][c] = e
        assert tables.tolist() == T0
        for src, dst, m in copies:
            k0[:, dst, :m], v0[:, dst, :m] = k0[:, src, :m].clone(), v0[:, src, :m].clone()
        assert torch.equal(kc, k0) and torch.equal(vc, v0)
        copied, gone_all = copied + taken, gone_all + gone
        free = torch.cat([free[taken:], dropped[:gone]])
        cached = lengths.clone()
        # every row's values lie where its table says
        p, t, was = parents.view(-1).tolist(), tokens.view(-1).tolist(), ended.view(-1).tolist()
        old, hist, new, flag = hist, [], [], []
        for r in range(rows):
            src = r // B * B + p[r]
            hist.append(list(old[src]))
            L = len(hist[r])
            assert want_len[r] == L
            at = torch.tensor([T0[r][i // page] * page + i % page for i in range(L)], device="cuda")
            for layer in range(layers):
                assert torch.equal(vc[layer].view(-1, hkv, d)[at], tok[layer][torch.tensor(hist[r], device="cuda")][:, hkv:])
            new.append([] if was[src] else [t[r]])
            hist[r] += new[r]
            flag.append(1 if was[src] else int(t[r] == end))
        scores, ended = new_scores, torch.tensor(flag, dtype=torch.uint8, device="cuda").view(n, B)
    assert bsm.bsm_device_status() == 0 and copied + gone_all > 0
