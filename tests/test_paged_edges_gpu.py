"""Paged attention where a key must take no part: pages that are not there, keys
a mask hides whose values are not finite, values near the end of the type's
range; and pages that several requests share.

The reference is the definition in 64 bits, the sum over the visible keys alone
(no product with a weight of 0).  Tolerances are those derived in
test_paged_gpu.py; infinities have to be equal and NaN has to meet NaN.
"""
import numpy as np
import pytest

from paper_2002_07062_gb300 import bsm
from test_paged_gpu import Batch, MASKS, _types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def setup():
    import torch
    import __graft_entry__ as g
    g.build()
    torch.cuda.set_device(0)
    bsm.bsm_device_status_clear()


def exact(b, causal=True, window=0):
    """out, lse, sum_j p_j |v_j| and the largest scale * sum_d |q_d k_d| of every row."""
    import torch
    T, hq, d = b.q.shape
    g, P = hq // b.hkv, b.page
    f64 = dict(dtype=torch.float64, device="cuda")
    out, mass = torch.zeros((T, hq, d), **f64), torch.zeros((T, hq, d), **f64)
    lse, size = torch.full((T, hq), -float("inf"), **f64), torch.zeros((T, hq), **f64)
    for r, L in enumerate(int(x) for x in b.lens):
        t0, t1 = int(b.starts[r]), int(b.starts[r + 1])
        if t0 == t1 or L == 0:
            continue
        ids = torch.from_numpy(np.array(b.tables[r][:-(-L // P)], np.int64)).cuda()
        there = (ids >= 0) & (ids < b.kc.shape[0])
        ids = torch.where(there, ids, 0)
        k, v = (c[ids].reshape(-1, b.hkv, d)[:L].double() for c in (b.kc, b.vc))
        there = there.repeat_interleave(P)[:L]
        k, v = (torch.where(there[:, None, None], z, 0.0) for z in (k, v))
        key = torch.arange(L, device="cuda")
        pos = L - (t1 - t0) + torch.arange(t1 - t0, device="cuda")
        see = there[None, :].expand(t1 - t0, L)
        if causal:
            see = see & (key[None, :] <= pos[:, None])
            if window:
                see = see & (key[None, :] > pos[:, None] - window)
        for h in range(hq):
            x = torch.where(see, b.q[t0:t1, h].double() @ k[:, h // g].t() * b.scale, -float("inf"))
            top = x.amax(1, keepdim=True)
            top = torch.where(top == -float("inf"), 0.0, top)
            e = torch.exp(x - top)
            s = e.sum(1, keepdim=True)
            p = e / torch.where(s == 0, 1.0, s)
            vh = v[:, h // g]
            good = torch.where(torch.isfinite(vh), vh, 0.0)
            o = p @ good
            for j in (~torch.isfinite(vh)).any(1).nonzero().view(-1).tolist():
                o += torch.where(see[:, j, None] & ~torch.isfinite(vh[j]), vh[j], 0.0)
            out[t0:t1, h], mass[t0:t1, h] = o, p @ good.abs()
            lse[t0:t1, h] = (top + torch.log(s))[:, 0]
            kf = torch.nan_to_num(k[:, h // g], 0.0, 0.0, 0.0)
            size[t0:t1, h] = (b.q[t0:t1, h].double().abs() @ kf.abs().t() * b.scale).amax(1)
    return out, lse, mass, size


def check(b, causal=True, window=0):
    import torch
    out, lse, mass, size = exact(b, causal, window)
    _, u, tiny = _types()[b.dtype]
    e = b.d * 2.0 ** -24 * size + 2.0 ** -20 * (1 + size)
    bound = (u + 2 * e[..., None]) * mass + u * out.abs() + tiny
    got = b.out.double()
    ok = (torch.isnan(out) & torch.isnan(got)) | (out == got) | ((got - out).abs() <= bound) & torch.isfinite(out)
    assert ok.all(), (int((~ok).sum()), (~ok).nonzero()[:4].tolist(), out[~ok][:4].tolist(), got[~ok][:4].tolist())
    ls = b.lse.double()
    ok = (torch.isnan(lse) & torch.isnan(ls)) | (lse == ls) | ((ls - lse).abs() <= 2 * e + 2.0 ** -22 * lse.abs())
    assert ok.all(), (int((~ok).sum()), (~ok).nonzero()[:4].tolist(), lse[~ok][:4].tolist(), ls[~ok][:4].tolist())


def run(b, hint, causal=True, window=0, status=0):
    """One call with the given hint (None: the true one) into outputs filled with 7; the status word after it."""
    import torch
    b.out.fill_(7.0)
    b.lse.fill_(7.0)
    b.scale = b.d ** -0.5
    most = int(b.fresh.max(initial=0))
    ws = torch.full((bsm.bsm_paged_workspace_bytes(b.hq, b.hkv, b.d, most),), 255, dtype=torch.uint8, device="cuda")
    bsm.bsm_paged_attention(b.q, b.kc, b.vc, b.out, *b.dev(), most if hint is None else hint, b.scale, ws,
                            flags=bsm.FLAG_CAUSAL if causal else 0, window=window, lse=b.lse)
    torch.cuda.synchronize()
    got = bsm.bsm_device_status()
    bsm.bsm_device_status_clear()
    assert got == status


HINTS = [1 << 20, 0]        # the tile kernel, the row kernel


GONE = {
    "whole rows a copy": dict(lens=[700, 300, 90, 513], fresh=[130, 300, 1, 3], hq=8, hkv=2, d=128, page=16),
    "halves apart": dict(lens=[700, 300, 90, 513], fresh=[130, 300, 1, 3], hq=8, hkv=2, d=64, page=16),
    "halves apart, f16": dict(lens=[500, 300, 90, 400], fresh=[130, 300, 1, 3], hq=6, hkv=2, d=80, page=32, dtype="f16"),
    "large pages": dict(lens=[1700, 900, 300, 513], fresh=[130, 300, 1, 3], hq=4, hkv=1, d=128, page=256),
    "odd pages": dict(lens=[300, 200, 90, 213], fresh=[130, 200, 1, 3], hq=4, hkv=2, d=96, page=3),
    "pages of 1": dict(lens=[300, 200, 90, 213], fresh=[130, 200, 1, 3], hq=4, hkv=2, d=128, page=1, dtype="f16"),
    "long": dict(lens=[20000, 300, 9000, 4000], fresh=[2, 40, 1, 1], hq=8, hkv=1, d=128, page=16),
}


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("mask", ["causal", "full", "window 300"])
@pytest.mark.parametrize("name", GONE)
def test_keys_on_missing_pages_take_no_part(name, mask, hint):
    """Page ids outside the cache, as a table has them where pages ran out: their keys have no weight, whatever the
    scores of the others; a request without any page gets zeros and -inf; the others' answers are the same bits."""
    import torch
    b = Batch(**GONE[name], seed=len(name))
    # scores of the keys that are there far below 0, the score of a key of zeros
    b.q.copy_(-b.q.abs())
    b.kc.copy_(b.kc.abs())
    b.poison()
    run(b, hint, **MASKS[mask])
    whole, lse = b.out.clone(), b.lse.clone()
    need = -(-b.lens // b.page)
    b.tables = b.tables.copy()
    b.tables[0, [0, need[0] // 2]] = [b.kc.shape[0], -1]
    b.tables[0, need[0] - 1:need[0]] = 1 << 30
    b.tables[2, :need[2]] = -1
    run(b, hint, status=bsm.DEV_BOUNDS, **MASKS[mask])
    check(b, **MASKS[mask])
    for r in (1, 3):
        rows = slice(int(b.starts[r]), int(b.starts[r + 1]))
        assert torch.equal(whole[rows].view(torch.int16), b.out[rows].view(torch.int16))
        assert torch.equal(lse[rows], b.lse[rows])
    rows = slice(int(b.starts[2]), int(b.starts[3]))
    assert not b.out[rows].any() and bool((b.lse[rows] == -float("inf")).all())


def test_pages_that_ran_out():
    """The step of a server whose pool is empty: tables writes -1, attention goes over the keys that have a page."""
    import torch
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    b = Batch([40, 90, 33], [8, 50, 1], 8, 2, 128, 16, seed=1)
    tab, st, ln = i32(b.tables), i32([0] * 4), i32([0] * 3)
    tab[0, 2:], tab[1, 3:], tab[2, 2:] = -7, -7, -7
    n = b.T
    slots, pos, own = torch.zeros(n, dtype=torch.int64, device="cuda"), i32([0] * n), i32([0] * n)
    info = torch.zeros(4, dtype=torch.int64, device="cuda")
    free = i32([int(b.tables[0, 2]), int(b.tables[1, 3])])
    bsm.bsm_paged_tables(i32(b.lens - b.fresh), i32(b.fresh), free, 16, tab, st, ln, slots, pos, own, info)
    assert info.tolist() == [59, 2, 3, bsm.PAGED_PAGES]
    k, v = torch.randn(n, 2, 128, device="cuda").bfloat16(), torch.randn(n, 2, 128, device="cuda").bfloat16()
    bsm.bsm_paged_write(k, v, b.kc, b.vc, slots)
    b.tables = tab.cpu().numpy()
    for hint in HINTS:
        run(b, hint, status=bsm.DEV_BOUNDS)
        check(b)


BAD = {
    "chunk": dict(lens=[700, 90], fresh=[300, 1], hq=8, hkv=2, d=128, page=16),
    "chunk, head size 64, f16": dict(lens=[700, 300], fresh=[300, 300], hq=4, hkv=4, d=64, page=64, dtype="f16"),
    "chunk, odd pages": dict(lens=[400, 90], fresh=[200, 1], hq=6, hkv=2, d=96, page=5),
    "a few tokens": dict(lens=[200, 41, 8, 77], fresh=[4, 7, 8, 1], hq=8, hkv=4, d=128, page=16),
    "a few tokens, head size 40, f16": dict(lens=[200, 41, 8], fresh=[4, 7, 8], hq=2, hkv=2, d=40, page=16, dtype="f16"),
    "long": dict(lens=[9000], fresh=[700], hq=4, hkv=1, d=128, page=16),
    "long, a few tokens": dict(lens=[30000, 500], fresh=[6, 3], hq=2, hkv=1, d=128, page=16),
    "more tokens than keys": dict(lens=[30, 5], fresh=[90, 8], hq=4, hkv=2, d=64, page=16),
}


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("mask", ["causal", "full", "window 37", "window 300"])
@pytest.mark.parametrize("name", BAD)
def test_values_of_hidden_keys_do_not_show(name, mask, hint):
    """Infinities and NaN among a request's own keys and values, at its last tokens and scattered: they show in the
    tokens that see them and in no other."""
    import torch
    b = Batch(**BAD[name], seed=len(name))
    rng = np.random.default_rng(len(name) + len(mask))
    bad = [float("inf"), -float("inf"), float("nan")]
    for r, (L, m) in enumerate(zip(b.lens.tolist(), b.fresh.tolist())):
        # the last tokens, whole rows and single columns; some of the tokens before; and a key
        places = [L - 1, L - 2, L - max(1, m // 2)] + rng.integers(max(0, L - m - 40), L, 3).tolist()
        for i, at in enumerate(x for x in places if x >= 0):
            page, row = int(b.tables[r, at // b.page]), at % b.page
            if i == 0:
                b.vc[page, row] = float("nan")
            else:
                b.vc[page, row, int(rng.integers(b.hkv)), int(rng.integers(b.d))] = bad[i % 3]
        if m > 1:
            at = L - 1
            b.kc[int(b.tables[r, at // b.page]), at % b.page, 0, 0] = float("nan")
    b.poison()
    run(b, hint, **MASKS[mask])
    check(b, **MASKS[mask])


@pytest.mark.parametrize("hint", HINTS)
def test_requests_of_nothing_but_nan(hint):
    import torch
    b = Batch([3000, 300, 50], [900, 20, 1], 8, 2, 128, 16, seed=3)
    for e in range(-(-3000 // 16)):
        b.kc[int(b.tables[0, e])] = float("nan")
        b.vc[int(b.tables[0, e])] = float("nan")
    b.poison()
    run(b, hint)
    check(b)


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("fresh", [1, 200, 300])
def test_large_values_under_growing_scores(fresh, hint):
    """A value near the end of bf16's range at a key whose score, in base 2, lies 7.9 above those of all steps before
    (many requests, so that a CTA has all steps of a tile): its weight is less than 1, and so must be what it is
    multiplied by."""
    import torch
    n = 40
    b = Batch([700] * n, [fresh] * 2 + [1] * (n - 2), 8, 8, 64, 16, seed=4)
    b.q.zero_()
    b.q[..., 0] = 1.0
    b.kc.zero_()
    b.vc.normal_()
    for r in range(n):
        for at in (300, 450, 600):
            page = int(b.tables[r, at // 16])
            b.kc[page, at % 16, :, 0] = 7.9 * 8 / 1.4426950408889634
            b.vc[page, at % 16, 0, 5] = 3e38 if at == 450 else 1.0
            b.vc[page, at % 16, 1, 9] = -2e38 if at == 600 else 1.0
    run(b, hint)
    check(b)


_FIRST = """
import torch
from paper_2002_07062_gb300 import bsm
torch.manual_seed(0)
ws = torch.zeros(bsm.bsm_paged_workspace_bytes(8, 2, 64, 60), dtype=torch.uint8, device="cuda")
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
cached, fresh, free = i32([0, 0]), i32([60, 33]), torch.randperm(16, device="cuda", dtype=torch.int32)
tab, st, ln, pos, own = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), i32([0] * 3), i32([0] * 2), i32([0] * 93), i32([0] * 93)
slots, info = torch.zeros(93, dtype=torch.int64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
q, k, v = (torch.randn(93, h, 64, device="cuda").bfloat16() for h in (8, 2, 2))
kc, vc = torch.zeros(2, 16, 16, 2, 64, device="cuda").bfloat16()
out = torch.zeros_like(q)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    s = torch.cuda.current_stream()
    bsm.bsm_paged_tables(cached, fresh, free, 16, tab, st, ln, slots, pos, own, info, stream=s)
    bsm.bsm_paged_write(k, v, kc, vc, slots, stream=s)
    bsm.bsm_paged_attention(q, kc, vc, out, st, ln, tab, 60, 0.125, ws, flags=bsm.FLAG_CAUSAL, stream=s)
graph.replay()
torch.cuda.synchronize()
for a, b in ((0, 60), (60, 93)):
    kk, vv = (z[a:b].double().repeat_interleave(4, 1) for z in (k, v))
    x = torch.einsum("ihd,jhd->hij", q[a:b].double(), kk) * 0.125
    x = x.masked_fill(torch.ones_like(x[0], dtype=torch.bool).triu(1), -float("inf"))
    ref = torch.einsum("hij,jhd->ihd", x.softmax(-1), vv)
    assert float((out[a:b] - ref).abs().max()) <= 3 * 2.0 ** -8 * float(vv.abs().max())
assert info.tolist() == [93, 7, 0, 0] and bsm.bsm_device_status() == 0
print("captured first")
"""


def test_first_launches_of_a_process_may_be_captured():
    """After bsm_paged_workspace_bytes the library's first launches can be a capture."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stderr[-2000:]


def test_write_reads_what_the_kernel_before_it_wrote():
    """Launches overlap: a write follows, without a pause, the kernel that makes its keys."""
    import torch
    T, H, d = 4096, 8, 128
    kc, vc = torch.zeros(2, T // 16, 16, H, d, device="cuda", dtype=torch.bfloat16)
    slots = torch.randperm(T, device="cuda")
    k, v, back = (torch.zeros(T, H, d, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    st = torch.cuda.current_stream()
    for i in range(1, 60):
        # what the second write reads, the first has stored (and lets the second start early)
        k.fill_(i)
        bsm.bsm_paged_write(k, k, back.view(T // 16, 16, H, d), v.view(T // 16, 16, H, d), slots, stream=st)
        bsm.bsm_paged_write(v, back, kc, vc, slots, stream=st)
        assert bool((kc == i).all()) and bool((vc == i).all()), i


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("d,page", [(128, 16), (64, 16), (128, 3)])
def test_requests_that_share_pages(d, page, hint):
    """A common prefix lies in the cache once: its pages stand in every request's table."""
    b = Batch([700, 650, 90, 480], [130, 1, 3, 300], 8, 2, d, page, seed=5)
    b.tables = b.tables.copy()
    b.tables[1, :400 // page] = b.tables[0, :400 // page]
    b.tables[3, :160 // page] = b.tables[0, :160 // page]
    b.tables[2, :90 // page] = b.tables[3, :90 // page]
    b.poison()
    for mask in ("causal", "window 300"):
        run(b, hint, **MASKS[mask])
        check(b, **MASKS[mask])


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("gone", [False, True])
def test_lse_beside_values_of_nothing_but_nan(gone, hint):
    """The values have no part in lse: it is right where all outputs are NaN, also with a page missing."""
    b = Batch([3000, 300, 50], [900, 20, 1], 8, 2, 128, 16, seed=7)
    for r in (0, 1):
        for e in range(-(-int(b.lens[r]) // 16)):
            b.vc[int(b.tables[r, e])] = float("nan")
    if gone:
        b.tables = b.tables.copy()
        b.tables[0, 2], b.tables[1, 1] = -1, -1
    run(b, hint, status=bsm.DEV_BOUNDS if gone else 0)
    check(b)
