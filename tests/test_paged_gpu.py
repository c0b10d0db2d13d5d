"""Paged-cache operators on the GPU against the 64-bit oracle.

Tables, slots and written caches are compared bit for bit.  Attention's
tolerance, from its arithmetic: probabilities and the output are rounded to
the type (unit roundoff u, half a unit in the last of 8 and 11
significant bits: 2^-8 bf16, 2^-11 f16), everything else is fp32 (w = 2^-24).  A score is a sum of d products,
|error| <= d w A with A = scale * sum |q_d k_d|, the exponent and its argument
add about 2^-20 (1 + |s|), so every probability is off by a relative 2 (d w A +
2^-20 (1 + A)) at most, the sum's error included, and
  |out - exact| <= (u + 2 e) sum p |v| + u |exact| + tiny,  e = d w A + 2^-20 (1 + A)
  |lse - exact| <= 2 e + 2^-22 |lse|.
"""
import numpy as np
import pytest

from oracle import paged_oracle as O
from paper_2002_07062_gb300 import bsm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def setup():
    import torch
    import __graft_entry__ as g
    g.build()
    torch.cuda.set_device(0)
    bsm.bsm_device_status_clear()


def _types():
    import torch
    return {"bf16": (torch.bfloat16, 2.0 ** -8, 1e-38), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -24)}


class Batch:
    """Requests with their pages scattered over a pool, q / k / v drawn from N(0, 1)."""

    def __init__(self, lens, fresh, hq, hkv, d, page, dtype="bf16", seed=0, layout="nhd", spare=5, pad=0, qscale=1.0):
        import torch
        self.lens, self.fresh = np.array(lens), np.array(fresh)
        self.hq, self.hkv, self.d, self.page, self.dtype = hq, hkv, d, page, dtype
        n = len(lens)
        rng = np.random.default_rng(seed)
        need = -(-self.lens // page)
        pages = int(need.sum()) + spare
        order = rng.permutation(pages).astype(np.int32)
        self.tables = np.full((n, max(1, int(need.max(initial=0))) + 2), 1 << 29, np.int32)
        at = 0
        for r in range(n):
            self.tables[r, :need[r]] = order[at:at + need[r]]
            at += need[r]
        self.starts = np.concatenate([[0], np.cumsum(self.fresh)]).astype(np.int32)
        self.T = int(self.starts[-1]) + pad
        t = _types()[dtype][0]
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.q = (new(self.T, hq, d) * qscale).to(t)
        if layout == "hnd":
            self.kc = new(pages, hkv, page, d).to(t).transpose(1, 2)
            self.vc = new(pages, hkv, page, d).to(t).transpose(1, 2)
        else:
            self.kc, self.vc = new(pages, page, hkv, d).to(t), new(pages, page, hkv, d).to(t)
        self.out = torch.full((self.T, hq, d), 7.0, device="cuda", dtype=t)
        self.lse = torch.full((self.T, hq), 7.0, device="cuda")

    def poison(self):
        """NaN in every place of the caches that no request owns."""
        import torch
        used = torch.zeros(self.kc.shape[:2], dtype=torch.bool, device="cuda")
        for r, L in enumerate(self.lens):
            for e in range(-(-int(L) // self.page)):
                used[int(self.tables[r, e]), :min(self.page, int(L) - e * self.page)] = True
        for c in (self.kc, self.vc):
            c[~used] = float("nan")

    def dev(self):
        import torch
        return [torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda() for x in (self.starts, self.lens, self.tables)]

    def run(self, causal=True, window=0, scale=None, max_new=None, stream=None, lse=True):
        import torch
        nb = bsm.bsm_paged_workspace_bytes(self.hq, self.hkv, self.d, int(self.fresh.max(initial=0)))
        ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")      # (NaN)
        self.scale = scale or self.d ** -0.5
        bsm.bsm_paged_attention(self.q, self.kc, self.vc, self.out, *self.dev(),
                                int(self.fresh.max(initial=0)) if max_new is None else max_new, self.scale, ws,
                                flags=bsm.FLAG_CAUSAL if causal else 0, window=window, lse=self.lse if lse else None,
                                stream=stream)
        torch.cuda.synchronize()
        assert bsm.bsm_device_status() == 0
        return self.out

    def check(self, causal=True, window=0):
        import torch
        out, lse, mass, size = O.attention(self.q, self.kc, self.vc, self.starts, self.lens, self.tables, self.scale,
                                           causal, window)
        T = int(self.starts[-1])
        _, u, tiny = _types()[self.dtype]
        e = self.d * 2.0 ** -24 * size + 2.0 ** -20 * (1 + size)
        bound = (u + 2 * e[..., None]) * mass + u * out.abs() + tiny
        err = (self.out.double() - out).abs()[:T]
        wrong = ~(err <= bound[:T])
        assert not wrong.any(), (int(wrong.sum()), wrong.nonzero()[:4].tolist(), float(err.max()))
        none = torch.isinf(lse)
        assert torch.equal(torch.isinf(self.lse[:T]) & (self.lse[:T] < 0), none[:T])
        le = (self.lse.double() - lse).abs()
        ok = none | (le <= 2 * e + 2.0 ** -22 * lse.abs())
        assert ok[:T].all(), float(le[:T][~none[:T]].max())
        assert bool((self.out[T:] == 7.0).all()) and bool((self.lse[T:] == 7.0).all())


CASES = {
    "one token, one key": dict(lens=[1], fresh=[1], hq=1, hkv=1, d=64, page=16),
    "decode": dict(lens=[5, 100, 1, 333, 16, 17], fresh=[1] * 6, hq=8, hkv=2, d=128, page=16),
    "decode, no shared heads": dict(lens=[70, 3], fresh=[1, 1], hq=6, hkv=6, d=64, page=8),
    "decode, one shared head of 16": dict(lens=[1000, 31], fresh=[1, 1], hq=16, hkv=1, d=128, page=64),
    "three heads to one": dict(lens=[129, 64], fresh=[1, 2], hq=9, hkv=3, d=96, page=16),
    "forty heads to one": dict(lens=[77, 300], fresh=[1, 3], hq=40, hkv=1, d=64, page=32),
    "seventy heads to one": dict(lens=[50], fresh=[2], hq=140, hkv=2, d=32, page=16),
    "two hundred heads to one": dict(lens=[150], fresh=[5], hq=200, hkv=1, d=64, page=16),
    "some bring nothing": dict(lens=[40, 50, 0, 60], fresh=[0, 1, 0, 4], hq=4, hkv=2, d=64, page=16),
    "more tokens than keys": dict(lens=[3, 0, 40], fresh=[9, 2, 50], hq=4, hkv=2, d=64, page=16),
    "a few tokens": dict(lens=[90, 41, 8], fresh=[4, 7, 8], hq=8, hkv=2, d=128, page=16),
    "a chunk": dict(lens=[500], fresh=[201], hq=8, hkv=2, d=128, page=16),
    "prompts": dict(lens=[300, 257, 1, 64], fresh=[300, 257, 1, 64], hq=4, hkv=2, d=64, page=64),
    "prompts, f16": dict(lens=[300, 129], fresh=[300, 100], hq=4, hkv=4, d=128, page=32, dtype="f16"),
    "mixed": dict(lens=[400, 700, 20, 513, 130], fresh=[1, 300, 1, 130, 2], hq=8, hkv=2, d=128, page=16),
    "head size 8": dict(lens=[100, 33], fresh=[1, 20], hq=4, hkv=2, d=8, page=16),
    "head size 40": dict(lens=[100, 300], fresh=[1, 140], hq=4, hkv=2, d=40, page=16),
    "head size 72": dict(lens=[100, 300], fresh=[1, 140], hq=4, hkv=2, d=72, page=16),
    "head size 80, f16": dict(lens=[200, 300], fresh=[3, 140], hq=10, hkv=2, d=80, page=16, dtype="f16"),
    "pages of 1": dict(lens=[100, 65], fresh=[1, 60], hq=4, hkv=2, d=64, page=1),
    "pages of 3": dict(lens=[100, 65], fresh=[1, 60], hq=4, hkv=2, d=128, page=3),
    "pages of 48": dict(lens=[100, 500], fresh=[1, 400], hq=4, hkv=2, d=128, page=48),
    "pages of 256": dict(lens=[100, 700], fresh=[1, 600], hq=4, hkv=2, d=128, page=256),
    "pages of 8": dict(lens=[9, 350], fresh=[1, 349], hq=4, hkv=2, d=128, page=8),
    "five heads to one, chunk": dict(lens=[260], fresh=[260], hq=10, hkv=2, d=128, page=16),
    "seven heads to one, chunk": dict(lens=[400], fresh=[150], hq=7, hkv=1, d=64, page=16),
    "long": dict(lens=[40000, 5], fresh=[1, 1], hq=8, hkv=2, d=128, page=32),
    "long, a few tokens": dict(lens=[30000], fresh=[6], hq=16, hkv=2, d=128, page=16, dtype="f16"),
    "heads in front of tokens": dict(lens=[300, 70], fresh=[150, 1], hq=8, hkv=2, d=128, page=16, layout="hnd"),
    "large scores": dict(lens=[300, 70], fresh=[150, 1], hq=8, hkv=2, d=128, page=16, qscale=20.0),
    "padded": dict(lens=[200, 70], fresh=[90, 1], hq=8, hkv=2, d=64, page=16, pad=37),
}
MASKS = {"causal": dict(causal=True), "full": dict(causal=False), "window 1": dict(causal=True, window=1),
         "window 37": dict(causal=True, window=37), "window 300": dict(causal=True, window=300)}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("name", CASES)
def test_attention(name, mask):
    b = Batch(**CASES[name], seed=len(name))
    b.poison()
    b.run(**MASKS[mask])
    b.check(**MASKS[mask])


LONG = {
    # several steps and tiles a CTA, both row blocks of a tile
    "tiles": dict(lens=[3000, 2500, 1800], fresh=[700, 1, 400], hq=16, hkv=8, d=128, page=16),
    "tiles, head size 64": dict(lens=[3100, 2500, 77], fresh=[900, 300, 1], hq=16, hkv=16, d=64, page=64),
    "tiles, f16": dict(lens=[2900, 2100], fresh=[333, 500], hq=24, hkv=8, d=128, page=32, dtype="f16"),
    # tiles of one row block: the key steps of both softmax groups
    "few rows": dict(lens=[60000, 33], fresh=[3, 5], hq=16, hkv=2, d=128, page=16),
    "few rows, head size 64, f16": dict(lens=[50000], fresh=[9], hq=16, hkv=4, d=64, page=128, dtype="f16"),
    "single tokens beside a prompt": dict(lens=[900 + 37 * i for i in range(20)] + [700], fresh=[1] * 20 + [700], hq=8,
                                          hkv=8, d=128, page=8),
    # the row kernel, several steps a warp
    "single tokens": dict(lens=[1 + 511 * i for i in range(30)], fresh=[1] * 30, hq=16, hkv=8, d=128, page=16),
    "single tokens, head size 64": dict(lens=[9000 - 511 * i for i in range(17)], fresh=[1] * 17, hq=12, hkv=4, d=64,
                                        page=48, dtype="f16"),
    # one tile in many parts
    "one token, one key/value head": dict(lens=[70000], fresh=[1], hq=16, hkv=1, d=128, page=16),
    "a few tokens, one key/value head": dict(lens=[20, 40000], fresh=[1, 3], hq=5, hkv=1, d=64, page=64, dtype="f16"),
    "40 tokens, one key/value head": dict(lens=[60000], fresh=[40], hq=4, hkv=1, d=64, page=16),
    "20 tokens beside others": dict(lens=[50000, 2000], fresh=[20, 1], hq=3, hkv=1, d=120, page=12, dtype="f16"),
    "prompts in pages of 4": dict(lens=[700, 900], fresh=[150, 1], hq=8, hkv=4, d=96, page=4),
}


@pytest.mark.parametrize("keys", ["even", "growing", "falling"])
@pytest.mark.parametrize("mask", ["causal", "full", "window 300"])
@pytest.mark.parametrize("name", LONG)
def test_long_runs(name, mask, keys):
    """Many steps a unit.  Keys that grow (or fall) along the request make every
    row's maximum rise step after step (or lie in its first step)."""
    import torch
    b = Batch(**LONG[name], seed=len(name) + len(mask))
    if keys != "even":
        for r, L in enumerate(b.lens):
            for e in range(-(-int(L) // b.page)):
                f = e * b.page / max(1, int(L))
                b.kc[int(b.tables[r, e])] *= 0.2 + 6 * (f if keys == "growing" else 1 - f)
    b.poison()
    b.run(**MASKS[mask])
    b.check(**MASKS[mask])


def test_drawn_batches():
    """Shapes drawn over the whole range, every mask and type."""
    rng = np.random.default_rng(11)
    for i in range(40):
        n = int(rng.integers(1, 9))
        fresh = np.where(rng.random(n) < 0.5, 1, rng.integers(0, 260, n))
        lens = np.maximum(0, fresh + rng.integers(-20, 900, n) * (rng.random(n) < 0.8))
        hkv, g = int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 3, 5, 8, 17, 33]))
        b = Batch(lens, fresh, hkv * g, hkv, int(rng.choice([8, 24, 64, 80, 112, 128])),
                  int(rng.choice([1, 2, 8, 16, 24, 64, 200])), dtype=str(rng.choice(["bf16", "f16"])), seed=100 + i,
                  layout=str(rng.choice(["nhd", "hnd"])), pad=int(rng.integers(0, 5)))
        if b.T == 0:
            continue
        m = MASKS[str(rng.choice(list(MASKS)))]
        b.poison()
        b.run(**m)
        b.check(**m)


def test_many_requests():
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 60, 3000)
    fresh = np.minimum(lens, rng.integers(0, 3, 3000))
    b = Batch(lens, fresh, 4, 2, 64, 16, seed=2)
    b.poison()
    b.run()
    b.check()


def test_hint_and_lse_do_not_change_the_answer():
    import torch
    b = Batch([300, 700, 20], [1, 150, 12], 8, 2, 128, 16, seed=3)
    b.run(max_new=0)
    b.check()
    b.run(max_new=1 << 20)
    b.check()
    b.run()
    first = b.out.clone()
    b.run(lse=False)
    assert torch.equal(first.view(torch.int16), b.out.view(torch.int16))


def test_same_answer_every_time():
    import torch
    b = Batch([5000, 700, 20, 1300], [1, 150, 12, 400], 8, 2, 128, 16, seed=4)
    b.run()
    first, lse = b.out.clone(), b.lse.clone()
    for _ in range(5):
        b.out.zero_()
        b.run()
        assert torch.equal(first.view(torch.int16), b.out.view(torch.int16)) and torch.equal(lse, b.lse)


def test_fused_projection_strides_and_strided_out():
    import torch
    b = Batch([300, 45], [130, 1], 8, 2, 64, 16, seed=5)
    qkv = torch.full((b.T, 12, 64), 3.0, device="cuda", dtype=b.q.dtype)
    qkv[:, :8] = b.q
    b.q = qkv[:, :8]
    wide = torch.full((b.T, 10, 64), 7.0, device="cuda", dtype=b.q.dtype)
    b.out = wide[:, 1:9]
    b.run()
    b.check()
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 9] == 7.0).all())
    # keys and values side by side in one allocation
    both = torch.stack([b.kc, b.vc], 1).contiguous()
    b.kc, b.vc = both[:, 0], both[:, 1]
    b.run()
    b.check()
    # heads outermost, pages between heads and tokens
    far = both.permute(1, 3, 0, 2, 4).contiguous()
    b.kc, b.vc = far[0].permute(1, 2, 0, 3), far[1].permute(1, 2, 0, 3)
    b.run()
    b.check()


@pytest.mark.parametrize("d,page", [(128, 16), (128, 8), (128, 256), (64, 16), (96, 32)])
@pytest.mark.parametrize("order", ["4 rows more a page", "8 rows more a page", "24 rows more a page", "pages inside tokens",
                                   "heads first", "one page", "a wider row"])
def test_cache_strides(order, d, page):
    """Caches whose pages lie whole groups of eight rows apart, or not."""
    import torch
    lens, fresh = ([page - 1], [page - 2]) if order == "one page" else ([700, 90, 2 * page], [300, 1, 40])
    b = Batch(lens=lens, fresh=fresh, hq=4, hkv=2, d=d, page=page, seed=d + page, spare=0 if order == "one page" else 3,
              qscale=2.0)
    for name in ("kc", "vc"):
        c = getattr(b, name)
        n = c.shape[0]
        if "more" in order:
            w = torch.full((n, page + int(order.split()[0]), 2, d), float("nan"), device="cuda", dtype=c.dtype)[:, :page]
        elif order == "pages inside tokens":
            w = torch.empty((page, n, 2, d), device="cuda", dtype=c.dtype).transpose(0, 1)
        elif order == "heads first":
            w = torch.empty((2, n, page, d), device="cuda", dtype=c.dtype).permute(1, 2, 0, 3)
        elif order == "a wider row":
            w = torch.full((n, page, 3, d + 8), float("nan"), device="cuda", dtype=c.dtype)[:, :, 1:, :d]
        else:
            w = torch.empty_like(c)
        w.copy_(c)
        setattr(b, name, w)
    b.poison()
    for mask in ("causal", "full", "window 300"):
        b.out.fill_(7.0)
        b.lse.fill_(7.0)
        b.run(**MASKS[mask])
        b.check(**MASKS[mask])


def test_tables_inside_a_wider_array():
    import torch
    b = Batch([300, 45, 700], [130, 1, 5], 8, 2, 64, 16, seed=8)
    st, ln, tab = b.dev()
    wide = torch.full((3, tab.shape[1] + 9), -1, dtype=torch.int32, device="cuda")
    wide[:, 4:4 + tab.shape[1]] = tab
    b.dev = lambda: [st, ln, wide[:, 4:4 + tab.shape[1]]]
    for hint in (130, 0):
        b.run(max_new=hint)
        b.check()


def test_two_streams_at_once():
    """Calls on two streams with a workspace each."""
    import torch
    bs = [Batch([5000, 700], [1, 400], 8, 2, 128, 16, seed=20), Batch([3000, 900, 4], [1, 1, 1], 8, 2, 128, 16, seed=21)]
    streams = [torch.cuda.Stream() for _ in bs]
    ws = [torch.full((bsm.bsm_paged_workspace_bytes(8, 2, 128, 400),), 255, dtype=torch.uint8, device="cuda") for _ in bs]
    args = [b.dev() for b in bs]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s, w, x in zip(bs, streams, ws, args):
            bsm.bsm_paged_attention(b.q, b.kc, b.vc, b.out, *x, int(b.fresh.max()), 128 ** -0.5, w, flags=bsm.FLAG_CAUSAL,
                                    lse=b.lse, stream=s)
    torch.cuda.synchronize()
    for b in bs:
        b.scale = 128 ** -0.5
        b.check()
    assert bsm.bsm_device_status() == 0


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes and 2^31 elements: the pages in use lie at its end."""
    import torch
    b = Batch([600, 41], [150, 1], 8, 2, 128, 16, seed=6)
    pages = (1 << 31) // (16 * 2 * 128) + 4096
    shift = pages - b.kc.shape[0]
    kc = torch.zeros((pages, 16, 2, 128), dtype=b.kc.dtype, device="cuda")
    vc = torch.zeros_like(kc)
    kc[shift:], vc[shift:] = b.kc, b.vc
    b.kc, b.vc = kc, vc
    b.tables = np.where(b.tables < 1 << 28, b.tables + shift, b.tables)
    b.run()
    b.check()
    slots = torch.tensor([pages * 16 - 1, -1, shift * 16], device="cuda")
    k = torch.randn(3, 2, 128, device="cuda").bfloat16()
    bsm.bsm_paged_write(k, k * 2, kc, vc, slots)
    torch.cuda.synchronize()
    assert torch.equal(kc[pages - 1, 15], k[0]) and torch.equal(vc[shift, 0], k[2] * 2)


def test_bad_tables_and_lengths_are_reported():
    """Ids and lengths outside the buffers: the kernels' own checks skip them and set the status bit."""
    import torch
    for case in ("page", "negative page", "length", "starts"):
        b = Batch([300, 80], [140, 1], 8, 2, 128, 16, seed=7)
        if case == "page":
            b.tables[0, 2] = b.kc.shape[0]
        if case == "negative page":
            b.tables[1, 1] = -5
        if case == "length":
            b.lens = np.array([300, b.tables.shape[1] * 16 + 1])
            b.tables[b.tables == 1 << 29] = 0
        if case == "starts":
            b.starts = np.array([0, 140, 170], np.int32)
        nb = bsm.bsm_paged_workspace_bytes(8, 2, 128, 140)
        ws = torch.zeros(nb, dtype=torch.uint8, device="cuda")
        for hint in (140, 0):           # the tile kernel, the row kernel
            bsm.bsm_paged_attention(b.q, b.kc, b.vc, b.out, *b.dev(), hint, 0.1, ws, flags=bsm.FLAG_CAUSAL)
            torch.cuda.synchronize()
            assert bsm.bsm_device_status() == bsm.DEV_BOUNDS, (case, hint)
            bsm.bsm_device_status_clear()


def _tables_case(cached, fresh, page, width=None, n_free=None, n_slots=None, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    cached, fresh = np.array(cached, np.int64), np.array(fresh, np.int64)
    have, need = -(-cached // page), -(-(cached + fresh) // page)
    width = width or max(1, int(need.max(initial=1)))
    total = int((need - have).sum())
    order = rng.permutation(int(need.sum()) + 50).astype(np.int32)
    tab = np.full((len(cached), width), -7, np.int32)
    at = 0
    for r in range(len(cached)):
        w = min(int(have[r]), width)
        tab[r, :w] = order[at:at + w]
        at += w
    free = order[at:at + (total + 9 if n_free is None else n_free)]
    n_slots = int(fresh.sum()) + 3 if n_slots is None else n_slots
    want = O.tables(cached.tolist(), fresh.tolist(), free.tolist(), page, tab, n_slots)
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    i32 = lambda n: torch.full((n,), -99, dtype=torch.int32, device="cuda")
    i64 = lambda n: torch.full((n,), -99, dtype=torch.int64, device="cuda")
    n = len(cached)
    got = [cu(tab), i32(n + 1), i32(n), i64(n_slots), i32(n_slots), i32(n_slots), i64(4)]
    for _ in range(2):          # the second call finds the first one's answer
        bsm.bsm_paged_tables(cu(cached), cu(fresh), cu(free), page, got[0], *got[1:])
    torch.cuda.synchronize()
    for name, g, w in zip(("tables", "starts", "lengths", "slots", "positions", "owners"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    info = got[6].tolist()
    assert info[:3] == list(want[6])
    return info[3]


@pytest.mark.parametrize("page", [1, 3, 16, 256])
@pytest.mark.parametrize("n,most_cached,most_fresh", [(1, 0, 1), (1, 5000, 3000), (7, 40, 2), (300, 900, 30),
                                                      (2048, 60, 3), (2049, 60, 3), (5000, 40, 9)])
def test_tables(n, most_cached, most_fresh, page):
    rng = np.random.default_rng(n + page)
    assert _tables_case(rng.integers(0, most_cached + 1, n), rng.integers(0, most_fresh + 1, n), page, seed=n) == 0


def test_tables_that_do_not_fit():
    assert _tables_case([30, 31, 32, 0], [1, 1, 1, 40], 16, n_free=2) == bsm.PAGED_PAGES
    assert _tables_case([30, 31, 32, 0], [1, 1, 1, 40], 16, n_free=0) == bsm.PAGED_PAGES
    assert _tables_case([30, 10], [5, 40], 16, width=2) == bsm.PAGED_WIDTH
    assert _tables_case([80, 10], [5, 4], 16, width=2) == bsm.PAGED_WIDTH
    assert _tables_case([30, 10], [5, 40], 16, n_slots=9) == bsm.PAGED_TOKENS
    assert _tables_case([30, 10], [5, 40], 16, n_slots=0) == bsm.PAGED_TOKENS


def test_tables_negative_lengths_and_none():
    import torch
    cu = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    tab, st, ln = torch.full((2, 4), -7, dtype=torch.int32, device="cuda"), cu([0] * 3), cu([0] * 2)
    sl, po, ow = torch.zeros(4, dtype=torch.int64, device="cuda"), cu([0] * 4), cu([0] * 4)
    info = torch.zeros(4, dtype=torch.int64, device="cuda")
    bsm.bsm_paged_tables(cu([-3, 2]), cu([2, -1]), cu([5, 6]), 16, tab, st, ln, sl, po, ow, info)
    assert info.tolist() == [2, 1, 0, bsm.PAGED_NEGATIVE]
    assert sl.tolist() == [80, 81, -1, -1] and st.tolist() == [0, 2, 2] and ln.tolist() == [2, 2]
    bsm.bsm_paged_tables(cu([]), cu([]), cu([5, 6]), 16, tab[:0], st, ln[:0], sl, po, ow, info)
    assert info.tolist() == [0, 0, 0, 0] and sl.tolist() == [-1] * 4 and st.tolist()[0] == 0


@pytest.mark.parametrize("layout", ["nhd", "hnd"])
@pytest.mark.parametrize("dtype,d", [("bfloat16", 128), ("float16", 72), ("float32", 4), ("float32", 80)])
@pytest.mark.parametrize("T,H,page", [(1, 1, 16), (37, 3, 16), (700, 8, 5)])
def test_write(T, H, page, dtype, d, layout):
    import torch
    t = getattr(torch, dtype)
    pages = T // page + 4
    g = torch.Generator(device="cuda").manual_seed(T + d)
    shape = (pages, page, H, d) if layout == "nhd" else (pages, H, page, d)
    kc, vc = [torch.randn(shape, generator=g, device="cuda").to(t) for _ in range(2)]
    if layout == "hnd":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    kv = torch.randn((T, 2 * H, d), generator=g, device="cuda").to(t)
    slots = torch.from_numpy(np.random.default_rng(T).permutation(pages * page)[:T].copy()).cuda()
    if T > 3:
        slots[[1, T - 1]] = -1
    want_k, want_v = kc.clone(), vc.clone()
    for i, s in enumerate(slots.tolist()):
        if s >= 0:
            want_k[s // page, s % page] = kv[i, :H]
            want_v[s // page, s % page] = kv[i, H:]
    bsm.bsm_paged_write(kv[:, :H], kv[:, H:], kc, vc, slots)
    torch.cuda.synchronize()
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)
    assert bsm.bsm_device_status() == 0


def test_write_past_the_cache_is_reported():
    import torch
    kc, vc = torch.zeros(4, 16, 2, 64, device="cuda").bfloat16(), torch.zeros(4, 16, 2, 64, device="cuda").bfloat16()
    k = torch.ones(2, 2, 64, device="cuda").bfloat16()
    bsm.bsm_paged_write(k, k, kc, vc, torch.tensor([64, 3], device="cuda"))
    torch.cuda.synchronize()
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS
    bsm.bsm_device_status_clear()
    assert float(kc.sum()) == 128.0 and bool((kc[0, 3] == 1).all())


def test_step_on_a_side_stream_and_in_a_graph():
    """Tables, write and attention in turn on a stream of their own, then captured once and replayed on new lengths."""
    import torch
    page, hq, hkv, d, n = 16, 8, 2, 64, 3
    pages, width, T = 64, 12, 40
    cached, fresh = torch.tensor([30, 0, 95], dtype=torch.int32, device="cuda"), \
        torch.tensor([1, 37, 2], dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, device="cuda", dtype=torch.int32)
    tab = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    tab[0, :2], tab[2, :6] = order[:2], order[2:8]
    free = order[8:].contiguous()
    i32 = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda")
    starts, lengths, pos, own = i32(n + 1), i32(n), i32(T), i32(T)
    slots, info = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    new = lambda *s: torch.randn(s, device="cuda").bfloat16()
    kc, vc, q, k, v = new(pages, page, hkv, d), new(pages, page, hkv, d), new(T, hq, d), new(T, hkv, d), new(T, hkv, d)
    out = torch.zeros_like(q)
    ws = torch.zeros(bsm.bsm_paged_workspace_bytes(hq, hkv, d, 38), dtype=torch.uint8, device="cuda")

    def step():
        st = torch.cuda.current_stream()
        bsm.bsm_paged_tables(cached, fresh, free, page, tab, starts, lengths, slots, pos, own, info, stream=st)
        bsm.bsm_paged_write(k, v, kc, vc, slots, stream=st)
        bsm.bsm_paged_attention(q, kc, vc, out, starts, lengths, tab, 38, d ** -0.5, ws, flags=bsm.FLAG_CAUSAL,
                                stream=st)

    def check(n_tok):
        torch.cuda.synchronize()
        assert int(info[0]) == n_tok and int(info[3]) == 0
        for t in range(n_tok):
            assert torch.equal(kc.view(-1, hkv, d)[slots[t]], k[t])
        ref, _, mass, size = O.attention(q, kc, vc, starts.tolist(), lengths.tolist(), tab.tolist(), d ** -0.5, True)
        e = d * 2.0 ** -24 * size + 2.0 ** -20 * (1 + size)
        bound = (2.0 ** -8 + 2 * e[..., None]) * mass + 2.0 ** -8 * ref.abs()
        assert ((out.double() - ref).abs() <= bound)[:n_tok].all()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    check(40)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    cached.copy_(torch.tensor([31, 37, 97], dtype=torch.int32))
    fresh.copy_(torch.tensor([1, 1, 20], dtype=torch.int32))
    free[:3] = free[-3:].clone()
    graph.replay()
    check(22)
    assert bsm.bsm_device_status() == 0


def test_serving_example():
    """The example's steps against its own recomputation: prompts in chunks, then single tokens, four layers.
    An output is a mean of values under rounded weights: half a unit of 8 bits twice, of the largest value."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import paged_serving
    worst = paged_serving.main(["--requests", "5", "--prompt", "300", "--chunk", "128", "--steps", "6", "--check"])
    assert worst <= 2 * 2.0 ** -8 * 4       # (means of values up to 4 times the largest output)
