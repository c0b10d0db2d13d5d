"""Refusals of the beam operators, without a GPU: every argument error comes back
before any CUDA call.  And the layout of their descriptors."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2002_07062_gb300 import bsm

INV, MIS, UNS = bsm.ERR_INVALID_ARG, bsm.ERR_MISALIGNED, bsm.ERR_UNSUPPORTED
AT = 1 << 40
# the device is asked for only after every argument has passed
PASSES = (bsm.ERR_NO_DEVICE, bsm.ERR_CUDA)
no_gpu = pytest.mark.skipif(__import__("torch").cuda.is_available(), reason="would launch on made-up addresses")


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()


def _fill(d, **kw):
    at = 1 << 32
    for name, ct in d._fields_:
        if ct is ctypes.c_void_p:
            setattr(d, name, at)
            at += 1 << 32
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _select(**kw):
    d = _fill(bsm.BeamSelectDesc(), **dict(dict(
        workspace_bytes=1 << 31, stride_request=4000, stride_beam=1000, n_requests=3, beams=4, vocab=1000, keep=8,
        end_token=2, dtype=bsm.BF16), **kw))
    return bsm.lib().bsm_beam_select(ctypes.addressof(d), None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_requests=-1), INV), (dict(beams=0), INV), (dict(vocab=0), INV), (dict(keep=0), INV), (dict(dtype=3), INV),
    (dict(stride_request=-1), INV), (dict(stride_beam=-1), INV), (dict(stride_request=1 << 60), INV),
    (dict(stride_beam=1 << 59), INV), (dict(end_token=-1), INV), (dict(end_token=1000), INV),
    (dict(beams=65), UNS), (dict(keep=65), UNS), (dict(vocab=(1 << 20) + 1), UNS), (dict(n_requests=1 << 22), UNS),
    (dict(logits=None), INV), (dict(scores=None), INV), (dict(out_scores=None), INV), (dict(parents=None), INV),
    (dict(tokens=None), INV), (dict(workspace=None), INV),
    (dict(logits=AT + 1), MIS), (dict(logits=AT + 2, dtype=bsm.F32), MIS), (dict(scores=AT + 2), MIS),
    (dict(out_scores=AT + 1), MIS), (dict(parents=AT + 2), MIS), (dict(tokens=AT + 2), MIS), (dict(workspace=AT + 128), MIS),
    (dict(parents=AT, tokens=AT + 92), INV), (dict(out_scores=AT, scores=AT + 44), INV), (dict(tokens=AT, ended=AT + 95), INV),
    (dict(logits=AT, workspace=AT + 23808), INV), (dict(workspace=AT, parents=AT + 4), INV),
    (dict(n_requests=0, logits=None), bsm.OK),
])
def test_select_refusals(kw, code):
    assert _select(**kw) == code


@no_gpu
@pytest.mark.parametrize("kw", [
    dict(), dict(ended=None, end_token=-5), dict(stride_request=0, stride_beam=0), dict(logits=AT + 2),
    dict(parents=AT, tokens=AT + 96, out_scores=AT + 192), dict(beams=64, keep=64, vocab=1 << 20),
    dict(logits=AT, workspace=AT + 24064),
])
def test_select_allowed(kw):
    assert _select(**kw) in PASSES


def _reorder(**kw):
    d = _fill(bsm.PagedReorderDesc(), **dict(dict(
        workspace_bytes=1 << 31, parent_stride=4, table_stride=10, new_table_stride=10, kv_stride_layer=0, kv_stride_page=2048,
        kv_stride_token=128, kv_stride_head=64, n_requests=3, beams=4, table_width=10, n_free=6, n_dropped=7, page_size=16,
        n_layers=1, n_pages=30, n_heads=2, head_dim=64, dtype=bsm.BF16), **kw))
    return bsm.lib().bsm_paged_reorder(ctypes.addressof(d), None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_requests=-1), INV), (dict(beams=0), INV), (dict(table_width=0), INV), (dict(n_free=-1), INV),
    (dict(n_dropped=-1), INV), (dict(page_size=0), INV), (dict(n_layers=0), INV), (dict(n_pages=0), INV), (dict(n_heads=0), INV),
    (dict(head_dim=0), INV), (dict(dtype=3), INV), (dict(parent_stride=-1), INV), (dict(table_stride=9), INV),
    (dict(new_table_stride=9), INV), (dict(table_stride=1 << 58), INV),
    (dict(beams=65), UNS), (dict(table_width=1 << 20, table_stride=1 << 20, new_table_stride=1 << 20), UNS),
    (dict(n_requests=1 << 30), UNS), (dict(page_size=1 << 30), UNS), (dict(n_layers=(1 << 20) + 1), UNS),
    (dict(parents=None), INV), (dict(lengths=None), INV), (dict(tables=None), INV), (dict(free_pages=None), INV),
    (dict(new_lengths=None), INV), (dict(new_tables=None), INV), (dict(dropped=None), INV), (dict(info=None), INV),
    (dict(k_cache=None), INV), (dict(v_cache=None), INV), (dict(workspace=None), INV),
    (dict(kv_stride_page=1024), INV), (dict(n_layers=2), INV), (dict(n_layers=2, kv_stride_layer=2048 * 29), INV),
    (dict(kv_stride_head=-64), INV),
    (dict(parents=AT + 2), MIS), (dict(tables=AT + 1), MIS), (dict(info=AT + 4), MIS), (dict(dropped=AT + 2), MIS),
    (dict(k_cache=AT + 8), MIS), (dict(workspace=AT + 16), MIS), (dict(head_dim=60), MIS),
    (dict(kv_stride_token=132, kv_stride_page=4096), MIS),
    (dict(lengths=AT, new_lengths=AT + 4), INV), (dict(tables=AT, new_tables=AT + 40), INV),
    (dict(tables=AT, new_tables=AT, new_table_stride=12), INV), (dict(new_lengths=AT, new_tables=AT), INV),
    (dict(dropped=AT, free_pages=AT + 20), INV), (dict(info=AT, parents=AT + 28), INV), (dict(k_cache=AT, v_cache=AT), INV),
    (dict(k_cache=AT, tables=AT + 512), INV), (dict(workspace=AT, v_cache=AT + 512), INV),
    (dict(lengths=AT, new_tables=AT), INV),
])
def test_reorder_refusals(kw, code):
    assert _reorder(**kw) == code


@no_gpu
@pytest.mark.parametrize("kw", [
    dict(), dict(lengths=AT, new_lengths=AT), dict(tables=AT, new_tables=AT), dict(n_free=0, free_pages=None),
    dict(n_dropped=0, dropped=None), dict(n_layers=3, kv_stride_layer=30 * 2048), dict(n_requests=0, parents=None, k_cache=None),
    dict(parent_stride=8), dict(parent_stride=0),
    # keys and values interleaved in one allocation, layers inside of pages
    dict(n_layers=2, kv_stride_page=8192, kv_stride_layer=4096, kv_stride_token=256, k_cache=AT, v_cache=AT + 256),
])
def test_reorder_allowed(kw):
    assert _reorder(**kw) in PASSES


def test_workspace_sizes_refused():
    for args in [(-1, 4, 10), (1, 0, 10), (1, 65, 10), (1, 4, 0), (1, 4, 1 << 20), (1 << 30, 4, 10)]:
        assert bsm.lib().bsm_paged_reorder_workspace_bytes(*args) == -1
        with pytest.raises(ValueError):
            bsm.bsm_paged_reorder_workspace_bytes(*args)
    assert bsm.bsm_paged_reorder_workspace_bytes(3, 4, 10) > 0

    for args in [(-1, 4, 100, 4), (1, 0, 100, 4), (1, 65, 100, 4), (1, 4, 0, 4), (1, 4, 100, 0), (1, 4, 100, 65),
                 (1, 4, (1 << 20) + 1, 4)]:
        assert bsm.lib().bsm_beam_select_workspace_bytes(-1, *args) == -1
        with pytest.raises(ValueError):
            bsm.bsm_beam_select_workspace_bytes(*args)


def test_null_descriptors_and_layout(tmp_path):
    assert bsm.lib().bsm_beam_select(None, None) == INV and bsm.lib().bsm_paged_reorder(None, None) == INV
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    for desc, name in ((bsm.BeamSelectDesc, "bsm_beam_select_desc"), (bsm.PagedReorderDesc, "bsm_paged_reorder_desc")):
        fields = [n for n, _ in desc._fields_]
        src = tmp_path / (name + ".c")
        src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "bsm.h"\nint main(void){printf("%%zu",sizeof(%s));'
                       % name + "".join('printf(" %%zu",offsetof(%s,%s));' % (name, n) for n in fields) + "return 0;}\n")
        exe = str(tmp_path / name)
        subprocess.run(["gcc", "-I", os.path.dirname(bsm.HEADER), str(src), "-o", exe], check=True)
        got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
        assert got == [ctypes.sizeof(desc)] + [getattr(desc, n).offset for n in fields]


def test_binding_refuses_tensors_the_library_cannot_see():
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)
    with pytest.raises(ValueError):
        bsm.bsm_beam_select(z(2, 3, 50), z(2, 3), z(2, 4), z(2, 4, dt=torch.int32), z(2, 4, dt=torch.int32),
                            z(64, dt=torch.uint8))
    i = lambda *s: z(*s, dt=torch.int32)
    with pytest.raises(ValueError):
        bsm.bsm_paged_reorder(i(2, 3), i(6), i(6, 4), i(5), i(6), i(6, 4), i(5), z(4, dt=torch.int64), z(4, 16, 2, 64),
                              z(4, 16, 2, 64), z(64, dt=torch.uint8))
