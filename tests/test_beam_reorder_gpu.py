"""The paged cache after beams were kept: tables, lengths, copied and dropped
pages against plain loops; and a whole decode step with beams."""
import math

import numpy as np
import pytest
import torch

from oracle import beam_oracle as O
from oracle import paged_oracle as OP
from paper_2002_07062_gb300 import bsm

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def clean_status():
    bsm.bsm_device_status_clear()
    yield
    torch.cuda.synchronize()
    bsm.bsm_device_status_clear()


def _i32(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Case:
    """Rows that share their first pages, as beams of one prompt do."""

    def __init__(self, n, B, page, lo, hi, prompt=0, layers=1, hkv=2, d=64, dtype="bf16", seed=0, width=None, equal=False,
                 layout="layers", spread=None, n_free=None):
        rng = np.random.default_rng(seed)
        self.n, self.B, self.page = n, B, page
        L = rng.integers(lo, hi + 1, (n, 1 if equal else B)) * np.ones((1, B), np.int64)
        L = np.maximum(L, prompt)
        shared, need = prompt // page, -(-L // page)
        self.width = width or int(need.max()) + 2
        pages = int(need.sum()) + n * B + 5
        order = rng.permutation(pages)
        nxt = 0
        t = rng.integers(-1, pages, (n, B, self.width))         # what lies past a row's length is not read
        for r in range(n):
            t[r, :, :shared] = order[nxt:nxt + shared]
            nxt += shared
            for b in range(B):
                k = int(need[r, b]) - shared
                t[r, b, shared:shared + k] = order[nxt:nxt + k]
                nxt += k
        self.free_h = order[nxt:nxt + (n * B if n_free is None else n_free)]
        self.lengths, self.tables, self.free = _i32(L.reshape(-1)), _i32(t.reshape(n * B, self.width)), _i32(self.free_h)
        self.parents = _i32(rng.integers(0, B, (n, B)) if spread is None else np.minimum(rng.geometric(spread, (n, B)) - 1, B - 1))
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(DT[dtype])
        if layout == "layers":
            self.k, self.v = (rnd(layers, pages, page, hkv, d) for _ in range(2))
        elif layout == "pages":                 # keys and values of all layers of a page together, heads outside of tokens
            both = rnd(pages, 2, layers, hkv, page, d)
            self.k, self.v = (both[:, i].permute(1, 0, 3, 2, 4) for i in (0, 1))
        self.dropped = torch.full((n * B * self.width,), -7, dtype=torch.int32, device="cuda")
        self.info = torch.full((4,), -7, dtype=torch.int64, device="cuda")
        self.ws = torch.full((bsm.bsm_paged_reorder_workspace_bytes(n, B, self.width),), 255, dtype=torch.uint8, device="cuda")

    def run(self, in_place=False, stream=None):
        self.new_lengths = self.lengths if in_place else torch.full_like(self.lengths, -9)
        self.new_tables = self.tables if in_place else torch.full_like(self.tables, -9)
        bsm.bsm_paged_reorder(self.parents, self.lengths, self.tables, self.free, self.new_lengths, self.new_tables,
                              self.dropped, self.info, self.k, self.v, self.ws, stream=stream)

    def check(self, in_place=False, flags=0):
        L, T, k0, v0 = self.lengths.clone(), self.tables.clone(), self.k.clone(), self.v.clone()
        cap = self.width * self.page
        length, tab, copies, missing, dropped = O.reorder(
            self.parents.tolist(), [min(max(x, 0), cap) for x in L.tolist()], T.tolist(), self.free.tolist(), self.page)
        self.run(in_place)
        torch.cuda.synchronize()
        assert self.new_lengths.tolist() == length
        want = (T if in_place else torch.full_like(T, -9)).cpu().numpy()
        for (i, c), e in tab.items():
            want[i, c] = e
        assert np.array_equal(self.new_tables.cpu().numpy(), want)
        assert self.info.tolist() == [len(copies), missing, len(dropped), flags]
        assert self.dropped.tolist() == dropped + [-7] * (self.dropped.numel() - len(dropped))
        for src, dst, m in copies:
            if max(src, dst) < self.k.shape[1]:
                k0[:, dst, :m], v0[:, dst, :m] = k0[:, src, :m].clone(), v0[:, src, :m].clone()
        assert torch.equal(self.k, k0) and torch.equal(self.v, v0)
        return self


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kw", [
    dict(n=1, B=1, page=16, lo=5, hi=5), dict(n=1, B=4, page=16, lo=30, hi=40, prompt=20),
    dict(n=64, B=5, page=16, lo=20, hi=200, prompt=20, layers=3), dict(n=3, B=64, page=8, lo=1, hi=60, d=8),
    dict(n=5, B=8, page=64, lo=64, hi=70, equal=True, layers=2, dtype="f32"), dict(n=2, B=3, page=1, lo=0, hi=300, prompt=100),
    dict(n=7, B=4, page=16, lo=32, hi=32), dict(n=300, B=2, page=16, lo=0, hi=50, d=8), dict(n=2, B=16, page=16, lo=3000, hi=9000, hkv=1, d=8),
    dict(n=600, B=3, page=4, lo=1, hi=9, d=16, dtype="f16"), dict(n=4, B=6, page=100, lo=1, hi=450, spread=0.6, layers=2),
    dict(n=2, B=4, page=16, lo=0, hi=0), dict(n=9, B=7, page=48, lo=10, hi=500, prompt=9, hkv=5, d=96)])
def test_tables_copies_and_dropped_pages(kw, in_place):
    Case(seed=len(kw), **kw).check(in_place)
    assert bsm.bsm_device_status() == 0


@pytest.mark.parametrize("layout", ["layers", "pages"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_strides(layout, dtype):
    Case(6, 4, 16, 1, 100, layers=5, hkv=3, d=40, dtype=dtype, layout=layout, seed=1).check()


def test_one_layer_without_its_dimension():
    c = Case(6, 4, 16, 17, 100, seed=2)
    d = Case(6, 4, 16, 17, 100, seed=2)
    d.k, d.v = d.k[0], d.v[0]
    c.check()
    d.run()
    assert torch.equal(c.k[0], d.k) and torch.equal(c.v[0], d.v) and torch.equal(c.new_tables, d.new_tables)


def test_all_children_of_one_beam_and_none_moved():
    c = Case(4, 8, 16, 100, 120, prompt=90, seed=3)
    c.parents[:] = 5
    c.check()
    assert c.info[0] + c.info[1] > 0
    c = Case(4, 8, 16, 100, 120, prompt=90, seed=3)
    c.parents[:] = torch.arange(8, device="cuda")
    c.check()
    assert c.info.tolist() == [0, 0, 0, 0] and torch.equal(c.k, Case(4, 8, 16, 100, 120, prompt=90, seed=3).k)


def test_rows_out_of_use_and_bad_parents():
    c = Case(3, 4, 16, 5, 60, seed=4)
    c.parents[0, 1] = -1
    c.parents[1] = -1
    c.check()
    assert bsm.bsm_device_status() == 0
    c.parents[2, 0] = 4
    c.check()
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS


def test_shared_tails_are_split_whoever_shares_them():
    c = Case(2, 4, 16, 40, 40, seed=5)
    c.tables[1], c.tables[2] = c.tables[0], c.tables[0]     # a prompt's rows as a program first lays them out
    c.parents[:] = torch.arange(4, device="cuda")
    c.check()
    assert c.info[0] == 2
    keys = [c.k[:, c.new_tables[i].long()].flatten(1, 2)[:, :40] for i in range(3)]
    assert torch.equal(keys[0], keys[1]) and torch.equal(keys[0], keys[2])
    assert len({int(c.new_tables[i, 2]) for i in range(4)}) == 4


@pytest.mark.parametrize("left", [0, 1, 5])
def test_pages_run_out(left):
    c = Case(4, 4, 16, 33, 47, seed=6, n_free=left)
    c.parents[:] = 0
    c.check(flags=bsm.PAGED_PAGES)
    assert c.info.tolist()[:2] == [left, 12 - left]


def test_more_dropped_pages_than_listed():
    c = Case(5, 4, 16, 50, 60, seed=7)
    c.parents[:] = 1
    want = Case(5, 4, 16, 50, 60, seed=7)
    want.parents[:] = 1
    want.check()
    c.dropped = torch.full((6,), -7, dtype=torch.int32, device="cuda")
    c.run()
    assert c.dropped.tolist() == want.dropped.tolist()[:6] and c.info.tolist()[2:] == [want.info[2], bsm.PAGED_DROPPED]
    c.dropped = c.dropped[:0]
    c.run()
    assert c.info.tolist()[2:] == [want.info[2], bsm.PAGED_DROPPED]


def test_more_than_2_31_dropped_pages_and_few_listed():
    # 33 requests whose 64 rows of 2^20 - 1 pages are all given up: 2.2e9 dropped pages, room for 10 (27 GB)
    n, B, width = 33, 64, (1 << 20) - 1
    assert n * B * width > (1 << 31) + 10
    tables = torch.arange(B, dtype=torch.int32, device="cuda")[:, None].repeat(n, width)
    new = torch.full((n * B, width), -9, dtype=torch.int32, device="cuda")
    lengths = torch.full((n * B,), width, dtype=torch.int32, device="cuda")
    new_lengths = torch.full_like(lengths, -9)
    k, v = (torch.ones((70, 1, 1, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dropped = torch.full((12,), -7, dtype=torch.int32, device="cuda")
    info = torch.full((4,), -7, dtype=torch.int64, device="cuda")
    ws = torch.empty(bsm.bsm_paged_reorder_workspace_bytes(n, B, width), dtype=torch.uint8, device="cuda")
    bsm.bsm_paged_reorder(torch.full((n, B), -1, dtype=torch.int32, device="cuda"), lengths, tables, _i32([1]), new_lengths, new,
                          dropped[:10], info, k, v, ws)
    assert info.tolist() == [0, 0, n * B * width, bsm.PAGED_DROPPED]
    assert dropped.tolist() == list(range(10)) + [-7, -7] and (new_lengths == 0).all()
    assert bool((new == -9).all()) and bsm.bsm_device_status() == 0


def test_lengths_and_pages_outside_the_buffers():
    c = Case(2, 3, 16, 40, 40, seed=8, width=4)
    c.parents[:] = _i32([[0, 0, 1], [2, 2, 2]])
    pages = c.k.shape[1]
    c.tables[0, 2] = pages                      # a last page that is not in the cache: handed on, not copied
    c.lengths[5] = 1 << 30                      # cut to the table: whole pages, nothing to copy
    c.lengths[4] = -3
    c.tables[5] = torch.arange(4, device="cuda")
    before = c.k.clone()
    c.run()
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS
    assert c.new_lengths.tolist() == [40, 40, 40, 64, 64, 64]
    assert c.new_tables[:2, 2].tolist() == [pages, pages] and c.new_tables[3:].tolist() == [[0, 1, 2, 3]] * 3
    assert c.info.tolist()[:2] == [0, 0] and torch.equal(c.k, before)
    bsm.bsm_device_status_clear()
    c = Case(1, 3, 16, 40, 40, seed=8)
    c.parents[:] = 0
    c.free[0] = pages + 100                     # a free page that is not there
    before = c.k.clone()
    c.run()
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS and int(c.new_tables[1, 2]) == pages + 100
    assert c.info[0] == 2 and torch.equal(c.k[:, int(c.new_tables[2, 2]), :8], before[:, int(c.tables[0, 2]), :8])


@pytest.mark.parametrize("bad", [-1, -2, -(1 << 31)])
def test_free_pages_with_negative_ids_are_reported(bad):
    c = Case(1, 3, 16, 40, 40, seed=8)
    c.parents[:] = 0
    c.free[0] = bad                             # (a list that was padded)
    k, v, second = c.k.clone(), c.v.clone(), int(c.free[1])
    c.run()
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS
    assert c.new_tables[:, 2].tolist() == [int(c.tables[0, 2]), bad, second] and c.info.tolist()[:2] == [2, 0]
    for x, before in ((c.k, k), (c.v, v)):      # the other copy is made, and no other byte changes
        before[:, second, :8] = before[:, int(c.tables[0, 2]), :8].clone()
        assert torch.equal(x, before)
    # one that is not taken does not matter
    bsm.bsm_device_status_clear()
    c = Case(1, 3, 16, 40, 40, seed=8, n_free=5)
    c.free[2:] = bad
    c.parents[:] = 0
    c.check()
    assert bsm.bsm_device_status() == 0


@pytest.mark.parametrize("bad", [-2, -(1 << 31)])
def test_last_pages_with_negative_ids_are_reported(bad):
    c = Case(1, 3, 16, 40, 40, seed=8)
    c.parents[:] = _i32([[0, 0, 1]])
    c.tables[0, 2] = bad
    before = c.k.clone()
    c.run()
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS and c.new_tables[:2, 2].tolist() == [bad, bad]
    assert c.info.tolist()[:2] == [0, 0] and torch.equal(c.k, before)
    # a page that was missing already is passed on without a report
    bsm.bsm_device_status_clear()
    c = Case(1, 3, 16, 40, 40, seed=8)
    c.parents[:] = 0
    c.tables[0, 2] = -1
    c.check()
    assert bsm.bsm_device_status() == 0 and (c.new_tables[:, 2] == -1).all()


def test_no_requests():
    c = Case(1, 2, 16, 5, 5)
    bsm.bsm_paged_reorder(c.parents[:0], c.lengths[:0], c.tables[:0], c.free, c.lengths[:0], c.tables[:0], c.dropped, c.info,
                          c.k, c.v, c.ws)
    assert c.info.tolist() == [0, 0, 0, 0]


def test_parents_as_the_selection_gives_them_and_strided_tables():
    c = Case(5, 4, 16, 20, 90, seed=9)
    wide = torch.zeros((5, 11), dtype=torch.int32, device="cuda")
    wide[:, 2:6] = c.parents
    c.parents = wide[:, 2:6]
    tab = torch.full((20, c.width + 5), -3, dtype=torch.int32, device="cuda")
    tab[:, :c.width] = c.tables
    c.tables = tab[:, :c.width]
    c.check(in_place=True)
    assert (tab[:, c.width:] == -3).all()


def test_captured_and_on_another_stream():
    bsm.bsm_paged_workspace_bytes(8, 2, 128, 1)
    c, ref = Case(8, 4, 16, 20, 200, seed=10, layers=2), Case(8, 4, 16, 20, 200, seed=10, layers=2)
    other = Case(3, 4, 8, 2, 50, seed=11)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(stream=torch.cuda.current_stream())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph.replay()
    with torch.cuda.stream(side):
        other.run(stream=side)
    graph.replay()                              # (out of place: the same answer again)
    torch.cuda.synchronize()
    ref.check()
    for a in ("k", "v", "new_tables", "new_lengths", "info"):
        assert torch.equal(getattr(c, a), getattr(ref, a)), a
    assert torch.equal(c.dropped, ref.dropped)
    # replayed on other parents
    c.parents.copy_(c.parents.flip(1))
    graph.replay()
    ref.parents = c.parents.clone()
    ref.dropped.copy_(c.dropped)
    ref.run()
    torch.cuda.synchronize()
    assert torch.equal(c.new_tables, ref.new_tables) and torch.equal(c.dropped, ref.dropped)


def test_pages_far_into_the_cache():
    # pages past 2^31 elements and 2^32 bytes
    pages, page, hkv, d = 70000, 16, 16, 128
    k, v = (torch.zeros((pages, page, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i32 = dict(dtype=torch.int32, device="cuda")
    tables = torch.tensor([[69999, 69990], [3, 5], [4, 6]], **i32)
    lengths, free = torch.tensor([20, 20, 20], **i32), torch.tensor([69950, 69951], **i32)
    k[69990, :4], v[69990, :4] = 2.0, 3.0
    dropped, info = torch.zeros(6, **i32), torch.zeros(4, dtype=torch.int64, device="cuda")
    ws = torch.empty(bsm.bsm_paged_reorder_workspace_bytes(1, 3, 2), dtype=torch.uint8, device="cuda")
    bsm.bsm_paged_reorder(torch.zeros((1, 3), **i32), lengths, tables, free, lengths, tables, dropped, info, k, v, ws)
    assert tables.tolist() == [[69999, 69990], [69999, 69950], [69999, 69951]] and info.tolist() == [2, 0, 4, 0]
    for p in (69950, 69951):
        assert (k[p, :4] == 2).all() and (v[p, :4] == 3).all() and (k[p, 4:] == 0).all()
    # and keys rotated to slots there
    slots = torch.tensor([69999 * page + 7, 1], dtype=torch.int64, device="cuda")
    new = torch.randn((2, hkv, d), device="cuda").bfloat16()
    table = torch.cat([torch.zeros((9, 32)), torch.ones((9, 32))], 1).cuda()        # a quarter turn
    bsm.bsm_paged_write_rotary(None, new, new, None, k, v, slots, torch.tensor([8, 0], **i32), table)
    assert torch.equal(k[69999, 7, :, :32], -new[0, :, 32:64]) and torch.equal(k[69999, 7, :, 32:64], new[0, :, :32])
    assert torch.equal(k[69999, 7, :, 64:], new[0, :, 64:]) and torch.equal(v[69999, 7], new[0]) and torch.equal(v[0, 1], new[1])
    assert bsm.bsm_device_status() == 0
