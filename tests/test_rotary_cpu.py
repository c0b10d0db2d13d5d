"""Refusals of the rotary write, without a GPU: every argument error comes back
before any CUDA call.  And the layout of its descriptor."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2002_07062_gb300 import bsm

INV, MIS, UNS = bsm.ERR_INVALID_ARG, bsm.ERR_MISALIGNED, bsm.ERR_UNSUPPORTED
AT = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()


def _desc(**kw):
    d = bsm.PagedWriteRotaryDesc()
    at = 1 << 32
    for name, ct in d._fields_:
        if ct is ctypes.c_void_p:
            setattr(d, name, at)
            at += 1 << 32
    base = dict(q_stride_token=256, q_stride_head=64, k_stride_token=128, k_stride_head=64, v_stride_token=128,
                v_stride_head=64, q_out_stride_token=256, q_out_stride_head=64, kv_stride_page=2048, kv_stride_token=128,
                kv_stride_head=64, table_stride=64, n_tokens=3, heads_q=4, heads_kv=2, head_dim=64, rotary_dim=64,
                n_positions=100, page_size=16, n_pages=10, dtype=bsm.BF16, flags=0)
    for k, v in dict(base, **kw).items():
        setattr(d, k, v)
    return d


def _rc(**kw):
    d = _desc(**kw)
    return bsm.lib().bsm_paged_write_rotary(ctypes.addressof(d), None)


# queries, keys and values as parts of one row of 8 heads: all strides 512 and 64
FUSED = dict(q=AT, q_stride_token=512, k=AT + 4 * 128, k_stride_token=512, v=AT + 6 * 128, v_stride_token=512)
# the device is asked for only after every argument has passed
PASSES = (bsm.ERR_NO_DEVICE, bsm.ERR_CUDA)


@pytest.mark.parametrize("kw,code", [
    (dict(n_tokens=-1), INV), (dict(heads_q=-1), INV), (dict(heads_kv=0), INV), (dict(head_dim=0), INV),
    (dict(rotary_dim=-2), INV), (dict(rotary_dim=66), INV), (dict(rotary_dim=31), INV), (dict(n_positions=-1), INV),
    (dict(page_size=0), INV), (dict(n_pages=0), INV), (dict(dtype=3), INV), (dict(flags=1), INV), (dict(flags=4), INV),
    (dict(table_stride=63), INV), (dict(table_stride=-64), INV),
    (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(q_out=None), INV), (dict(k_cache=None), INV),
    (dict(table=None), INV), (dict(positions=None), INV), (dict(slots=None), INV),
    (dict(q_stride_token=128), INV), (dict(k_stride_token=64), INV), (dict(q_out_stride_head=0), INV),
    (dict(kv_stride_page=1024), INV), (dict(kv_stride_page=1 << 60), INV),
    (dict(q=AT + 8), MIS), (dict(q_out=AT + 8), MIS), (dict(k=AT + 2), MIS), (dict(v_stride_token=132), MIS),
    (dict(kv_stride_token=130, kv_stride_page=4096), MIS), (dict(slots=AT + 4), MIS), (dict(positions=AT + 2), MIS),
    (dict(table=AT + 2), MIS), (dict(head_dim=60, rotary_dim=60), MIS),
    (dict(heads_q=1024, q_stride_token=1 << 16, q_out_stride_token=1 << 16), UNS),
    (dict(k_cache=AT, v_cache=AT), INV), (dict(k=AT, k_cache=AT + 256), INV), (dict(q_out=AT, v_cache=AT + 64), INV),
    (dict(table=AT, k_cache=AT), INV), (dict(q_out=AT, table=AT + 64), INV), (dict(q_out=AT, positions=AT), INV),
    (dict(q=AT, q_out=AT + 128), INV),                              # q_out over other rows of q
    (dict(q=AT, q_out=AT, q_out_stride_token=320), INV),            # in place with other strides
    (dict(k=AT, q_out=AT), INV), (dict(v=AT, q_out=AT + 128), INV),
    (dict(FUSED, q_out=AT + 128, q_out_stride_token=512), INV),     # shifted onto its neighbours
    (dict(FUSED, q_out=AT + 64 * 2 * 2, q_out_stride_token=512), INV),
    (dict(FUSED, q_out=AT, q_out_stride_token=512, k=AT + 3 * 128), INV),
    (dict(n_tokens=0, k=None), bsm.OK),
])
def test_refusals(kw, code):
    assert _rc(**kw) == code


@pytest.mark.skipif(__import__("torch").cuda.is_available(), reason="would launch on made-up addresses")
@pytest.mark.parametrize("kw", [
    dict(), dict(heads_q=0, q=None, q_out=None), dict(rotary_dim=0, table=None), dict(rotary_dim=0, n_positions=0, table=None),
    dict(FUSED, q_out=AT, q_out_stride_token=512),                  # in place beside k and v
    dict(q=AT, q_out=AT), dict(n_tokens=1, q_stride_token=3, q=AT, q_out=AT),
    dict(q=AT, q_out=AT + 256 * 2, q_stride_token=512, q_out_stride_token=512),     # rows in one another's gaps
    dict(n_positions=1, table_stride=0), dict(head_dim=64, rotary_dim=18), dict(table=AT + 4, table_stride=65),
])
def test_allowed(kw):
    assert _rc(**kw) in PASSES


def test_null_descriptor_and_layout(tmp_path):
    assert bsm.lib().bsm_paged_write_rotary(None, None) == INV
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    names = [n for n, _ in bsm.PagedWriteRotaryDesc._fields_]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "bsm.h"\nint main(void){printf("%zu",sizeof('
                   'bsm_paged_write_rotary_desc));' + "".join(
                       'printf(" %%zu",offsetof(bsm_paged_write_rotary_desc,%s));' % n for n in names) + "return 0;}\n")
    exe = str(tmp_path / "t")
    subprocess.run(["gcc", "-I", os.path.dirname(bsm.HEADER), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(bsm.PagedWriteRotaryDesc)] + [getattr(bsm.PagedWriteRotaryDesc, n).offset for n in names]


def test_binding_refuses_tensors_the_library_cannot_see():
    import torch
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    with pytest.raises(ValueError):
        bsm.bsm_paged_write_rotary(z(3, 4, 64), z(3, 2, 64), z(3, 2, 64), z(3, 4, 64), z(4, 16, 2, 64), z(4, 16, 2, 64),
                                   z(3, dt=torch.int64), z(3, dt=torch.int32), z(9, 64, dt=torch.float32))
