"""Keys, values and queries rotated on the way to a paged cache, against the
definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import beam_oracle as O
from paper_2002_07062_gb300 import bsm

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def clean_status():
    bsm.bsm_device_status_clear()
    yield
    torch.cuda.synchronize()
    bsm.bsm_device_status_clear()


def _table(n, rot, far=0):
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    a = (far + torch.arange(n, dtype=torch.float64, device="cuda"))[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


def _close(got, ref, size, what):
    """fp32 arithmetic: each of two products and their sum is off by at most 2^-24 of the sizes that
    meet there; then one rounding to the output's type (half a step; below its normal numbers half of
    the smallest)."""
    e = torch.finfo(got.dtype)
    tol = e.eps / 2 * ref.abs() * (1 + 2.0 ** -20) + 3 * 2.0 ** -24 * size + e.tiny * e.eps / 2
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], ref[bad][:4])


def _case(T, hq, hkv, d, rot, inter, dtype, page=16, pages=None, n_pos=500, seed=0, layout="fused"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(DT[dtype])
    pages = pages or (T + page - 1) // page + 3
    if layout == "fused":               # parts of one row
        qkv = rnd(T, hq + 2 * hkv, d)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:                               # heads outside, tokens inside
        q, k, v = (rnd(h, T + 1, d).transpose(0, 1)[:T] for h in (hq, hkv, hkv))
    rng = np.random.default_rng(seed)
    slots = torch.from_numpy(rng.permutation(pages * page)[:T].astype(np.int64)).cuda()
    pos = torch.from_numpy(rng.integers(0, n_pos, T).astype(np.int32)).cuda()
    shape = (pages, page, hkv, d)
    if layout == "fused":
        kc, vc = rnd(*shape), rnd(*shape)
    else:                               # heads outside of pages, both caches in one allocation
        both = rnd(hkv, pages, 2, page, d)
        kc, vc = (both[:, :, i].permute(1, 2, 0, 3) for i in (0, 1))
    return q, k, v, kc, vc, slots, pos, _table(n_pos, rot)


def _check(q, k, v, kc, vc, slots, pos, table, inter, q_out=None, stream=None):
    kc0, vc0, q0, k0, v0 = kc.clone(), vc.clone(), q.clone(), k.clone(), v.clone()
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda") if q_out is None else q_out
    before = out.clone()
    bsm.bsm_paged_write_rotary(q, k, v, out, kc, vc, slots, pos, table, flags=bsm.FLAG_INTERLEAVED if inter else 0,
                               stream=stream)
    torch.cuda.synchronize()
    rot, P = table.shape[1], kc.shape[1]
    live = (pos >= 0) & (pos < table.shape[0])
    ref, size = O.rotary(q0, pos.tolist(), table, inter)
    assert torch.equal(out[~live], before[~live])
    _close(out[live], ref[live], size[live], "q_out")
    assert torch.equal(out[live][..., rot:], q0[live][..., rot:])
    ref, size = O.rotary(k0, pos.tolist(), table, inter)
    put = live & (slots >= 0) & (slots < kc.shape[0] * P)
    at = slots[put]
    _close(kc[at // P, at % P], ref[put], size[put], "k_cache")
    assert torch.equal(kc[at // P, at % P][..., rot:], k0[put][..., rot:])
    assert torch.equal(vc[at // P, at % P], v0[put])
    rest = torch.ones(kc.shape[:2], dtype=torch.bool, device="cuda")
    rest[at // P, at % P] = False
    assert torch.equal(kc[rest], kc0[rest]) and torch.equal(vc[rest], vc0[rest])
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32), (80, 80), (96, 20), (128, 18), (64, 2), (64, 0), (8, 6), (256, 256)])
def test_types_and_widths(dtype, inter, d, rot):
    _check(*_case(37, 6, 2, d, rot, inter, dtype, seed=d + rot), inter)
    assert bsm.bsm_device_status() == 0


@pytest.mark.parametrize("T,hq,hkv,page,layout", [
    (1, 32, 8, 16, "fused"), (1, 1, 1, 1, "heads"), (2, 3, 3, 5, "heads"), (300, 15, 5, 48, "fused"),
    (1000, 32, 8, 64, "heads"), (700, 7, 1, 16, "fused"), (129, 4, 4, 100, "heads")])
@pytest.mark.parametrize("inter", [False, True])
def test_shapes_and_strides(T, hq, hkv, page, layout, inter):
    _check(*_case(T, hq, hkv, 64, 64, inter, "bf16", page=page, layout=layout, seed=T), inter)
    assert bsm.bsm_device_status() == 0


@pytest.mark.parametrize("T", [3, 600])
def test_padding_tokens_without_slots_and_bounds(T):
    q, k, v, kc, vc, slots, pos, table = _case(T, 4, 2, 64, 64, False, "bf16", seed=5)
    pos[T // 2] = -1                        # padding: nothing of it is touched
    slots[T - 1] = -1                       # no page: its query is rotated all the same
    _check(q, k, v, kc, vc, slots, pos, table, False)
    assert bsm.bsm_device_status() == 0
    pos[0] = table.shape[0]                 # past the table
    _check(q, k, v, kc, vc, slots, pos, table, False)
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS
    bsm.bsm_device_status_clear()
    pos[0] = 3
    slots[0] = kc.shape[0] * kc.shape[1]    # past the cache
    _check(q, k, v, kc, vc, slots, pos, table, False)
    assert bsm.bsm_device_status() == bsm.DEV_BOUNDS


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T", [5, 800])
def test_queries_in_place_beside_keys_and_values(T, inter):
    q, k, v, kc, vc, slots, pos, table = _case(T, 8, 2, 128, 64, inter, "bf16", seed=T)
    _check(q, k, v, kc, vc, slots, pos, table, inter, q_out=q)


def test_without_queries_or_positions():
    q, k, v, kc, vc, slots, pos, table = _case(40, 4, 2, 64, 64, False, "f32", seed=1)
    ref, size = O.rotary(k, pos.tolist(), table, False)
    bsm.bsm_paged_write_rotary(None, k, v, None, kc, vc, slots, pos, table)
    _close(kc[slots // 16, slots % 16], ref, size, "k_cache")
    assert torch.equal(vc[slots // 16, slots % 16], v)
    before = kc.clone()
    bsm.bsm_paged_write_rotary(None, k, v, None, kc, vc, slots, pos, table[:0])     # no position is in the table
    torch.cuda.synchronize()
    assert torch.equal(kc, before) and bsm.bsm_device_status() == bsm.DEV_BOUNDS


def test_queries_come_with_a_place_to_go():
    q, k, v, kc, vc, slots, pos, table = _case(4, 4, 2, 64, 64, False, "bf16", seed=9)
    with pytest.raises(ValueError):
        bsm.bsm_paged_write_rotary(q, k, v, None, kc, vc, slots, pos, table)
    with pytest.raises(ValueError):
        bsm.bsm_paged_write_rotary(None, k, v, torch.empty_like(q), kc, vc, slots, pos, table)


def test_rotation_of_nothing_is_the_plain_write():
    q, k, v, kc, vc, slots, pos, table = _case(500, 4, 2, 64, 0, False, "bf16", seed=2)
    k2, v2 = kc.clone(), vc.clone()
    pos[:] = 1 << 20                        # (every position will do)
    bsm.bsm_paged_write_rotary(q, k, v, torch.empty_like(q), kc, vc, slots, pos, table)
    bsm.bsm_paged_write(k, v, k2, v2, slots)
    assert torch.equal(kc, k2) and torch.equal(vc, v2) and bsm.bsm_device_status() == 0


def test_table_of_odd_stride_and_address():
    q, k, v, kc, vc, slots, pos, table = _case(300, 4, 2, 64, 64, False, "bf16", seed=3)
    wide = torch.zeros((table.shape[0], 67), device="cuda")
    wide[:, 1:65] = table
    _check(q, k, v, kc, vc, slots, pos, wide[:, 1:65], False)
    _check(q, k, v, kc, vc, slots, pos, wide[:, 1:65], True)


def test_infinities_and_nans_stay_in_their_pair():
    q, k, v, kc, vc, slots, pos, table = _case(20, 4, 2, 64, 32, False, "f16", seed=4)
    k[3, 1, 5], q[7, 0, 40], v[2, 0, 3] = float("inf"), float("nan"), float("nan")
    bsm.bsm_paged_write_rotary(q, k, v, torch.empty_like(q), kc, vc, slots, pos, table)
    got = kc[slots // 16, slots % 16]
    bad = ~torch.isfinite(got)
    assert set(map(tuple, bad.nonzero().tolist())) <= {(3, 1, 5), (3, 1, 21)} and bad[3, 1].any()
    assert torch.equal(vc[slots // 16, slots % 16].view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot", [2, 18, 20, 30])
def test_columns_that_are_not_rotated_keep_their_bits(dtype, inter, rot):
    # NaNs of every kind beside the last pair, in queries and keys
    q, k, v, kc, vc, slots, pos, table = _case(40, 4, 2, 64, rot, inter, dtype, seed=rot)
    bits = torch.int32 if dtype == "f32" else torch.int16
    nans = {"bf16": [0x7fb1, 0x7f81, 0xff81 - 65536, 0xffc5 - 65536], "f16": [0x7d01, 0x7e55, 0xfc01 - 65536, 0xff33 - 65536],
            "f32": [0x7f800123, 0x7fc00345, 0xff800001 - (1 << 32), 0xffc0ffee - (1 << 32)]}[dtype]
    for x in (q, k):
        some = torch.tensor(nans, dtype=bits, device="cuda")[torch.arange(64 - rot, device="cuda") % 4]
        x.view(bits)[::2, :, rot:] = some
        assert torch.isnan(x[::2, :, rot:]).all()
    out = torch.empty_like(q)
    bsm.bsm_paged_write_rotary(q, k, v, out, kc, vc, slots, pos, table, flags=bsm.FLAG_INTERLEAVED if inter else 0)
    got = kc[slots // 16, slots % 16]
    assert torch.equal(out.view(bits)[..., rot:], q.view(bits)[..., rot:])
    assert torch.equal(got.view(bits)[..., rot:], k.view(bits)[..., rot:])
    for x, src in ((out, q), (got, k)):
        ref, size = O.rotary(src, pos.tolist(), table, inter)
        _close(x[..., :rot], ref[..., :rot], size[..., :rot], "rotated columns")


def test_captured_and_on_two_streams():
    a = _case(600, 8, 2, 128, 128, False, "bf16", seed=6)
    b = _case(3, 8, 2, 128, 128, True, "bf16", seed=7)
    outs = [torch.zeros_like(a[0]), torch.zeros_like(b[0])]
    bsm.bsm_paged_workspace_bytes(8, 2, 128, 1)         # (sets the library up)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph):
        bsm.bsm_paged_write_rotary(*a[:3], outs[0], *a[3:], stream=torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bsm.bsm_paged_write_rotary(*b[:3], outs[1], *b[3:], flags=bsm.FLAG_INTERLEAVED, stream=side)
    graph.replay()
    a[0].mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    for (q, _, _, _, _, _, pos, table), out, inter in ((a, outs[0], False), (b, outs[1], True)):
        ref, size = O.rotary(q, pos.tolist(), table, inter)
        _close(out, ref, size, "q_out")
