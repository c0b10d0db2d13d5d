"""Refusals of the paged-cache operators that need no GPU: tensors of several
devices, caches that overlap, counts and scales past what the kernels hold; and
layouts that must not be refused."""
import ctypes

import pytest
import torch

from paper_2002_07062_gb300 import bsm
from test_paged_cpu import INV, UNS, _attention, _tables, _write, built  # noqa: F401


class On:
    """A CPU tensor that says it lies on a GPU."""

    is_cuda = True

    def __init__(self, t, device=0):
        self._t, self._device = t, device

    def __getattr__(self, name):
        return getattr(self._t, name)

    def get_device(self):
        return self._device

    @property
    def device(self):
        return "cuda:%d" % self._device


class Library:
    """Takes every call and answers OK."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*a):
            self.calls += 1
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(bsm, "lib", lambda: lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return lib


I32 = dict(dtype=torch.int32)


def _args(name):
    half = lambda *s: On(torch.zeros(s, dtype=torch.bfloat16))
    i32 = lambda *s: On(torch.zeros(s, **I32))
    i64 = lambda *s: On(torch.zeros(s, dtype=torch.int64))
    if name == "tables":
        return dict(cached=i32(3), fresh=i32(3), free_pages=i32(9), page_size=16, tables=i32(3, 4), starts=i32(4),
                    lengths=i32(3), slots=i64(5), positions=i32(5), owners=i32(5), info=i64(4))
    if name == "write":
        return dict(k=half(5, 2, 64), v=half(5, 2, 64), k_cache=half(9, 16, 2, 64), v_cache=half(9, 16, 2, 64),
                    slots=i64(5))
    return dict(q=half(5, 4, 64), k_cache=half(9, 16, 2, 64), v_cache=half(9, 16, 2, 64), out=half(5, 4, 64),
                starts=i32(4), lengths=i32(3), tables=i32(3, 4), max_new=2, scale=0.125,
                workspace=On(torch.zeros(4096, dtype=torch.uint8)), lse=On(torch.zeros(5, 4)))


CALLS = {"tables": bsm.bsm_paged_tables, "write": bsm.bsm_paged_write, "attention": bsm.bsm_paged_attention}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_one_current_device(name, library, monkeypatch):
    """Every tensor of a call lies on the current device: the library launches there with bare addresses."""
    args = _args(name)
    CALLS[name](**args)
    assert library.calls == 1
    for key, value in args.items():
        if not isinstance(value, On):
            continue
        value._device = 1
        with pytest.raises(ValueError, match="cuda:1"):
            CALLS[name](**args)
        value._device = 0
    for value in args.values():
        if isinstance(value, On):
            value._device = 1
    with pytest.raises(ValueError, match="cuda:1"):
        CALLS[name](**args)
    assert library.calls == 1
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    CALLS[name](**args)
    assert library.calls == 2


@pytest.mark.parametrize("name", ["write", "attention"])
def test_strides_of_single_entries_do_not_matter(name, library):
    """Keys and values with one head, or one page: the stride of that dimension is never used and may differ."""
    args = _args(name)
    args["k_cache"] = On(torch.zeros(1, 16, 3, 64, dtype=torch.bfloat16)[:, :, :1])
    args["v_cache"] = On(torch.as_strided(args["k_cache"]._t, (1, 16, 1, 64), (5, 192, 8, 1)))
    for key in ("k", "v"):
        if key in args:
            args[key] = On(torch.zeros(5, 1, 64, dtype=torch.bfloat16))
    CALLS[name](**args)
    assert library.calls == 1
    args["v_cache"] = On(torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="same shape and strides"):
        CALLS[name](**args)


@pytest.fixture
def no_device():
    """These calls pass bare addresses that nothing lies at: one that is not refused must stop for want of a device."""
    if torch.cuda.is_available():
        pytest.skip("a call that is not refused would be launched")


def _write_code(**kw):
    d = _write(**kw)        # (kept until the call is over)
    return bsm.lib().bsm_paged_write(ctypes.addressof(d), None)


# pages of 16 tokens, 2 heads of 64 bf16: strides 2048, 128, 64 elements
@pytest.mark.parametrize("delta,strides,clash", [
    (64, {}, True),                             # values begin at the keys' second head
    (128, {}, True), (2048, {}, True), (9 * 2048, {}, True),            # second token, second page, last page
    (-64, {}, True), (-9 * 2048 - 15 * 128 - 64, {}, True),
    (10 * 2048, {}, False), (-10 * 2048, {}, False),                    # one behind the other
    (2048, dict(kv_stride_page=4096), False), (4096, dict(kv_stride_page=4096), True),      # pages in turn
    (6144, dict(kv_stride_page=4096), False),                           # ... three apart
    (64, dict(kv_stride_token=256, kv_stride_head=128, kv_stride_page=4096), False),        # rows in turn
    (32, dict(kv_stride_token=256, kv_stride_head=128, kv_stride_page=4096), True),         # ... half a row
    (128, dict(kv_stride_token=256, kv_stride_page=4096), False),       # all heads of a token, then the values'
    (10 * 64, dict(kv_stride_head=10 * 64 * 16, kv_stride_page=64, kv_stride_token=640), True),
    (20 * 64 * 16, dict(kv_stride_head=10 * 64 * 16, kv_stride_page=64, kv_stride_token=640), False),
])
def test_caches_that_share_a_place_are_refused(delta, strides, clash, no_device):
    """Keys and values may lie in one another's gaps; a place of both would get either."""
    at = 1 << 44
    code = _write_code(k_cache=at, v_cache=at + 2 * delta, **strides)
    assert (code == INV) == clash, code


def test_caches_that_share_a_place_against_counting(no_device):
    import random
    rng = random.Random(5)
    for _ in range(400):
        n = dict(page=rng.randint(1, 4), token=rng.randint(1, 4), head=rng.randint(1, 3))
        stride, cur = {}, 8
        for k in rng.sample(list(n), 3):
            stride[k] = cur + 8 * rng.choice([0, 0, 1, 2, 8])
            cur = stride[k] * n[k]
        places = {p * stride["page"] + t * stride["token"] + h * stride["head"] + x
                  for p in range(n["page"]) for t in range(n["token"]) for h in range(n["head"]) for x in range(8)}
        delta = 8 * rng.randint(-cur // 8 - 1, cur // 8 + 1)
        at = 1 << 44
        code = _write_code(k_cache=at, v_cache=at + 2 * delta, n_heads=n["head"], head_dim=8, page_size=n["token"],
                           n_pages=n["page"], kv_stride_page=stride["page"], kv_stride_token=stride["token"],
                           kv_stride_head=stride["head"], k_stride_token=8 * n["head"], k_stride_head=8,
                           v_stride_token=8 * n["head"], v_stride_head=8)
        assert (code == INV) == any(x + delta in places for x in places), (n, stride, delta, code)


@pytest.mark.parametrize("scale,refused", [(2.3e38, False), (2.4e38, True), (3.4e38, True), (1e-45, False)])
def test_scales_that_the_kernels_cannot_hold(scale, refused, no_device):
    """Scores are computed in base 2: scale * log2(e) has to be finite too."""
    d = _attention(scale=scale)
    assert (bsm.lib().bsm_paged_attention(ctypes.addressof(d), None) == INV) == refused


@pytest.mark.parametrize("make,call,field", [(_tables, "bsm_paged_tables", "n_requests"),
                                             (_attention, "bsm_paged_attention", "n_requests"),
                                             (_attention, "bsm_paged_attention", "n_tokens")])
def test_counts_that_32_bits_cannot_step_over(make, call, field, no_device):
    """Requests are scanned and tokens tiled in blocks: a count whose last block ends past 2^31 is refused before any
    launch (its loops would wrap)."""
    most = (1 << 31) - 1 - 4095
    for n, refused in ((most, False), (most + 1, True), ((1 << 31) - 1, True)):
        d = make(**{field: n})
        assert (getattr(bsm.lib(), call)(ctypes.addressof(d), None) == UNS) == refused, n
