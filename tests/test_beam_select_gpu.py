"""Continuations selected over beams and vocabulary, against the definition in
64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import beam_oracle as O
from paper_2002_07062_gb300 import bsm

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NEG = -float("inf")


def _tol(V, v):
    """The sum's terms: 2^-22 of the exponential and, for its argument (a difference and a product, half a
    step each, and log2(e) in fp32), 3 x 2^-24 of its size, whose mean under the softmax is at most log V, and
    4 more where the reference lags; what was summed before the reference moved is multiplied by such
    an exponential (by less than e^-4 each time: all of them together count as 1.02), once more at the end of a
    warp and of a part, and the parts by one of 2 x 2^-24.  Additions of half a step: 4 of a piece, one
    for each of V / 2048 pieces at most, 5 over a warp.  And the value's own rounding."""
    return 2.0 ** -24 * (4.1 * (4 + 3 * (math.log(V + 1) + 4)) + 2 + 9 + V / 2048 + np.abs(v))


def _run(logits, scores, keep, ended=None, end_token=0, stream=None, ws=None):
    n, B, V = logits.shape
    i32 = dict(dtype=torch.int32, device="cuda")
    out = [torch.full((n, keep), 7.0, device="cuda"), torch.full((n, keep), 77, **i32), torch.full((n, keep), 77, **i32)]
    if ws is None:
        ws = torch.full((bsm.bsm_beam_select_workspace_bytes(n, B, V, keep),), 255, dtype=torch.uint8, device="cuda")
    bsm.bsm_beam_select(logits, scores, *out, ws, ended=ended, end_token=end_token, stream=stream)
    return out


def _check(logits, scores, keep, ended=None, end_token=0, got=None):
    out = got or _run(logits, scores, keep, ended, end_token)
    torch.cuda.synchronize()
    V = logits.shape[2]
    val, par, tok = O.select(logits.double().cpu().numpy(), scores.cpu().numpy(), keep + 1,
                             None if ended is None else ended.cpu().numpy(), end_token)
    # beams' candidates that are apart, but by less than both tolerances, may come in either order
    with np.errstate(invalid="ignore"):
        gap = val[:, :-1] - val[:, 1:]
        close = (gap > 0) & np.isfinite(gap) & (gap <= 2 * _tol(V, val[:, 1:])) & (par[:, :-1] != par[:, 1:])
    near = close.copy()
    near[:, 1:] |= close[:, :-1]
    val, par, tok = val[:, :keep], par[:, :keep], tok[:, :keep]
    v, p, t = (x.cpu().numpy() for x in out)
    fin = np.isfinite(val)
    assert np.array_equal(np.isfinite(v), fin)
    assert (np.abs(v[fin] - val[fin]) <= _tol(V, val[fin])).all()
    same = (p == par) & (t == tok)
    assert (same | near).all(), (v[~same][:8], val[~same][:8], p[~same][:8], par[~same][:8], t[~same][:8], tok[~same][:8])
    assert near.mean() < 0.05
    return out


def _data(n, B, V, dtype, seed=0, scale=2.5, gap=0, off=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = (torch.randn(off + n * B * (V + gap), generator=g, device="cuda") * scale).to(DT[dtype])
    x = flat[off:].view(n, B, V + gap)[:, :, :V]
    s = -torch.rand((n, B), generator=g, device="cuda").cumsum(1) * 2 - 3
    return x, s


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,B,V,keep", [
    (1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 7, 4), (1, 4, 32000, 8), (3, 2, 513, 5), (5, 5, 4097, 10), (1, 1, 20000, 64),
    (2, 64, 300, 64), (40, 8, 1000, 16), (2, 4, 50001, 33), (1, 2, 200001, 12), (7, 1, 16385, 1), (200, 3, 129, 6)])
def test_types_and_sizes(dtype, n, B, V, keep):
    _check(*_data(n, B, V, dtype, seed=V), keep)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("gap,off", [(0, 1), (1, 0), (3, 5), (8, 7), (64, 0), (5, 2)])
def test_addresses_and_strides(dtype, gap, off):
    _check(*_data(3, 4, 9001, dtype, seed=gap + off, gap=gap, off=off), 9)


def test_rows_at_any_address_give_the_same_bits():
    row = (torch.randn(30001, device="cuda") * 3).bfloat16()
    outs = []
    for off in range(9):
        flat = torch.zeros(30001 + 16, device="cuda").bfloat16()
        flat[off:off + 30001] = row
        outs.append(_run(flat[off:off + 30001].view(1, 1, -1), torch.tensor([[-1.5]], device="cuda"), 20))
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("keep", [1, 6, 40, 64])
@pytest.mark.parametrize("V", [50, 5000, 40000])
def test_equal_values_go_by_beam_then_token(dtype, keep, V):
    x = torch.zeros((2, 3, V), device="cuda").to(DT[dtype])
    s = torch.tensor([[-1.0, -1.0, -1.0], [-2.0, -1.0, -2.0]], device="cuda")
    out = _check(x, s, keep)
    order = [(b, t) for b in range(3) for t in range(min(V, keep))][:keep]
    assert list(zip(out[1][0].tolist(), out[2][0].tolist()))[:keep] == order[:keep]
    # a few levels only, many ties at each; -0 and 0 are equal
    x = (torch.randint(0, 3, (2, 3, V), device="cuda") - 1.0).to(DT[dtype])
    x[0, 0, ::7] = -0.0
    _check(x, s + torch.tensor([0.0, -0.37, -0.81], device="cuda"), keep)


def test_equal_beams_tie_exactly():
    row = torch.randn(50001, device="cuda") * 2
    x = row.expand(1, 4, 50001)                     # one row for all beams, stride 0
    s = torch.full((1, 4), -2.25, device="cuda")
    v, p, t = _run(x, s, 8)
    assert p[0].tolist() == [0, 1, 2, 3] * 2 and len(set(t[0, :4].tolist())) == 1 and len(set(t[0, 4:].tolist())) == 1
    assert torch.equal(v[0, :4], v[0, :1].expand(4))
    v, p, t = _run(x.contiguous(), s, 8)            # the same values at four different alignments
    assert p[0].tolist() == [0, 1, 2, 3] * 2
    # and of a batch that all SMs share
    v, p, t = _run(row.expand(60, 4, 50001).contiguous(), torch.full((60, 4), -2.25, device="cuda"), 8)
    assert p.tolist() == [[0, 1, 2, 3] * 2] * 60 and (t == t[0]).all() and (v == v[0]).all()


def test_few_values_in_a_part_and_long_lists():
    # the last part of a row with fewer values than groups, values that all reach the bound, allowed tokens side by side
    _check(*_data(40, 4, 16384 * 2 + 9, "bf16", seed=21), 16)
    x, s = _data(12, 3, 30000, "bf16", seed=22)
    x[:, :, :20000], x[:, :, 21500:] = NEG, NEG
    _check(x, s, 30)
    _check(torch.zeros((9, 64, 700), device="cuda"), s[:9, :1].expand(9, 64).contiguous() - torch.arange(64, device="cuda") / 16, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 33000])
def test_order_within_ascending_and_descending_rows(dtype, V):
    up = torch.linspace(-4, 4, V, device="cuda").to(DT[dtype])
    x = torch.stack([up, up.flip(0)]).view(1, 2, V)
    _check(x, torch.tensor([[-0.5, -0.7]], device="cuda"), 20)


@pytest.mark.parametrize("V", [60, 9000, 120000])
@pytest.mark.parametrize("n", [1, 12])
def test_tokens_of_a_beam_follow_logits_that_lie_close(n, V):
    # 1e-12 apart beside a maximum of 5 and a logarithm below 13: more than 2^-44 of the largest
    assert 1e-12 > 2.0 ** -44 * 13
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.full((n, 1, V), -20.0, device="cuda")
    for r in range(n):
        at = torch.randperm(V, generator=g, device="cuda")[:41]
        x[r, 0, at[0]] = 5.0
        x[r, 0, at[1:]] = (torch.arange(40, device="cuda") - 20) * 1e-12
    _check(x, torch.full((n, 1), -0.75, device="cuda"), 30)


def test_beams_without_a_score():
    x, s = _data(4, 4, 3000, "bf16", seed=3)
    s[0, 1:] = NEG                                  # the first step: one beam
    s[1, :] = NEG                                   # nothing in use
    s[2, 0], s[2, 1] = float("nan"), float("inf")
    x[0, 2] = float("nan")                          # (never read)
    out = _check(x, s, 8)
    assert (out[1][1] == -1).all() and (out[2][1] == -1).all() and (out[0][1] == NEG).all()
    assert (out[1][0] == 0).all() and (out[1][2] >= 2).all()


@pytest.mark.parametrize("kind", [torch.bool, torch.uint8])
def test_finished_beams(kind):
    x, s = _data(6, 4, 700, "f32", seed=4)
    ended = torch.zeros((6, 4), dtype=kind, device="cuda")
    ended[0, 1] = ended[2, :] = ended[3, 0] = 1
    s[3, 0] = NEG                                   # finished and out of use
    x[2] = float("nan")
    out = _check(x, s, 10, ended, 699)
    assert sorted(out[1][2].tolist()) == [-1] * 6 + [0, 1, 2, 3] and set(out[2][2].tolist()) == {699, -1}
    assert torch.equal(out[0][2, :4], s[2].sort(descending=True).values)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_forbidden_tokens(dtype):
    x, s = _data(5, 3, 40000, dtype, seed=5)
    x[0, :, 5:] = NEG                               # a handful allowed
    x[1, 0] = NEG                                   # a row with nothing
    x[2, :, :] = NEG
    x[2, 1, 39999] = 3.0                            # one token of the request
    x[3, :, 1000:2000] = NEG
    x[4, :, :39000] = torch.finfo(DT[dtype]).min    # masked by the type's lowest value
    out = _check(x, s, 20)
    assert out[1][2].tolist() == [1] + [-1] * 19 and out[2][2, 0] == 39999
    assert abs(float(out[0][2, 0] - s[2, 1])) < 1e-6
    assert (out[1][0] >= 0).sum() == 15


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_of_the_lowest_value_are_uniform(dtype):
    x = torch.full((1, 2, 1000), torch.finfo(DT[dtype]).min, device="cuda", dtype=DT[dtype])
    out = _check(x, torch.tensor([[-1.0, -2.0]], device="cuda"), 4)
    assert out[2][0].tolist() == [0, 1, 2, 3] and out[1][0].tolist() == [0] * 4
    assert abs(float(out[0][0, 0]) + 1 + math.log(1000)) < 1e-4


def test_rows_with_nan_or_infinity_have_no_candidates():
    x, s = _data(3, 3, 20000, "f32", seed=6)
    x[0, 1, 19999] = float("nan")
    x[0, 2, 3] = float("inf")
    x[1, :, 7] = float("nan")
    x[2, 0, :] = float("nan")
    out = _check(x, s, 6)
    assert (out[1][0] == 0).all() and (out[1][1] == -1).all() and (out[1][2] > 0).all()


def test_infinity_beside_the_largest_f16_value():
    x, s = _data(2, 2, 700, "f16", seed=12)
    x[0, 0, 3], x[0, 0, 650] = 65504.0, float("inf")
    x[1, 0, 3] = 65504.0
    out = _check(x, s, 5)
    assert (out[1][0] == 1).all() and out[2][1, 0] == 3


def test_large_and_far_values():
    x, s = _data(2, 3, 6000, "f32", seed=7)
    x[0] *= 1e4                                     # one token has all the mass
    x[1] = x[1] * 1e30
    s[1] = -1e5
    _check(x, s, 12)


@pytest.mark.parametrize("dtype,at,step", [
    ("bf16", 1032, 8), ("bf16", -1032, 8), ("bf16", 508, 2), ("f16", 8200, 8), ("f16", -8200, 8), ("f16", 4100, 4), ("f32", 2 ** 26, 8)])
def test_values_about_as_far_apart_as_their_type_resolves(dtype, at, step):
    # the reference of the exponentials lags 4 at most where at + 4 is no number of the type, too
    g = torch.Generator(device="cuda").manual_seed(abs(at))
    x = at + step * (torch.rand((2, 3, 40001), generator=g, device="cuda") < 0.5).double()
    x[:, :, :17000] = at                                # (the larger value comes late)
    assert torch.equal(x.to(DT[dtype]).double(), x)
    s = torch.tensor([[-1.0, -1.3, -2.0], [-3.0, -1.0, -9.0]], device="cuda")
    out = _check(x.to(DT[dtype]), s, 7)
    count = (x[0, 0] == at + step).sum()
    want = -1 - math.log(int(count) + (40001 - int(count)) * math.exp(-step))
    assert abs(float(out[0][0, 0]) - want) <= _tol(40001, abs(want))


def test_sums_of_long_rows_by_their_own_formula():
    x, s = _data(1, 2, 1 << 20, "f32", seed=8)
    v, p, t = _check(x, s, 4)
    logp = torch.log_softmax(x.double(), -1) + s.double()[..., None]
    assert torch.allclose(v.double()[0], logp.view(-1).topk(4).values, atol=5e-6, rtol=0)


def test_captured_on_another_stream_and_side_by_side():
    x, s = _data(6, 4, 32000, "bf16", seed=9)
    y, z = _data(1, 2, 700, "f32", seed=10)
    bsm.bsm_paged_workspace_bytes(8, 2, 128, 1)
    ws = torch.empty(bsm.bsm_beam_select_workspace_bytes(6, 4, 32000, 8), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _run(x, s, 8, stream=torch.cuda.current_stream(), ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        with torch.cuda.stream(side):
            other = _run(y, z, 5, stream=side)
    torch.cuda.synchronize()
    _check(x, s, 8, got=got)
    _check(y, z, 5, got=other)
    first = [o.clone() for o in got]
    x.copy_(_data(6, 4, 32000, "bf16", seed=11)[0])
    graph.replay()
    _check(x, s, 8, got=got)
    x.copy_(_data(6, 4, 32000, "bf16", seed=9)[0])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_workspace_of_the_most_requests_serves_fewer():
    ws = torch.empty(bsm.bsm_beam_select_workspace_bytes(40, 4, 50001, 8), dtype=torch.uint8, device="cuda")
    for n, V in ((40, 50001), (9, 200000), (12, 50001), (8, 100), (1, 400000)):
        x, s = _data(n, 4, V, "bf16", seed=n)
        _check(x, s, 8, got=_run(x, s, 8, ws=ws))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,B,V", [(1, 1, 1 << 20), (1, 2, 1 << 20), (2, 3, 700001), (9, 1, 300000)])
def test_most_lists_of_the_most_kept_in_two_launches(dtype, n, B, V):
    # up to 128 lists of 64 entries join: random rows, rows that rise or fall (every part has the largest of the
    # parts before it below it), few levels (ties over all parts)
    x, s = _data(n, B, V, dtype, seed=B)
    _check(x, s, 64)
    up = torch.linspace(-6, 6, V, device="cuda").to(DT[dtype])
    _check(torch.stack([up, up.flip(0), up])[:B].expand(n, B, V).contiguous(), s, 64)
    _check((torch.randint(0, 2, (n, B, V), device="cuda") * 0.5).to(DT[dtype]), s, 64)
    # the 64 best one by one in different parts
    x[:] = -9.0
    at = (torch.arange(64, device="cuda") * (V // 64) + 11) % V
    x[:, :, at] = torch.arange(64, device="cuda").flip(0).to(DT[dtype]) * 0.125
    _check(x, s, 64)


def test_rows_far_apart():
    # more than 2^31 elements and 2^32 bytes from row to row
    far = 1_500_000_007
    flat = torch.zeros(3 * far + 3000, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((2, 2, 2500), (2 * far - 5, far, 1))
    x.copy_(_data(2, 2, 2500, "bf16", seed=30)[0])
    _check(x, torch.tensor([[-1.0, -1.3], [-0.2, -2.0]], device="cuda"), 7)
