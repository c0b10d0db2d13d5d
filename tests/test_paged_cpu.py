"""Refusals of the paged-cache operators, without a GPU: every argument error
comes back before any CUDA call.  And the layout of their descriptors."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2002_07062_gb300 import bsm


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


def _tables(**kw):
    return _fill(bsm.PagedTablesDesc(), **dict(dict(table_stride=8, n_requests=4, n_free=9, page_size=16, table_width=8,
                                                    n_slots=5), **kw))


def _write(**kw):
    return _fill(bsm.PagedWriteDesc(), **dict(dict(
        k_stride_token=128, k_stride_head=64, v_stride_token=128, v_stride_head=64, kv_stride_page=2048,
        kv_stride_token=128, kv_stride_head=64, n_tokens=3, n_heads=2, head_dim=64, page_size=16, n_pages=10,
        dtype=bsm.BF16), **kw))


def _attention(**kw):
    return _fill(bsm.PagedDesc(), **dict(dict(
        workspace_bytes=1 << 31, q_stride_token=256, q_stride_head=64, out_stride_token=256, out_stride_head=64,
        kv_stride_page=2048, kv_stride_token=128, kv_stride_head=64, table_stride=8, n_requests=2, n_tokens=3, heads_q=4,
        heads_kv=2, head_dim=64, page_size=16, n_pages=10, table_width=8, max_new=2, dtype=bsm.BF16, window=0,
        flags=bsm.FLAG_CAUSAL, scale=0.125), **kw))


INV, MIS, UNS = bsm.ERR_INVALID_ARG, bsm.ERR_MISALIGNED, bsm.ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,code", [
    (dict(n_requests=-1), INV), (dict(n_free=-1), INV), (dict(page_size=0), INV), (dict(table_width=0), INV),
    (dict(n_slots=-1), INV), (dict(table_stride=7), INV), (dict(table_width=1 << 20, table_stride=1 << 20), UNS), (dict(starts=None), INV), (dict(info=None), INV),
    (dict(cached=None), INV), (dict(fresh=None), INV), (dict(tables=None), INV), (dict(lengths=None), INV),
    (dict(free_pages=None), INV), (dict(slots=None), INV), (dict(owners=None), INV),
    (dict(slots=(1 << 40) + 4), MIS), (dict(cached=(1 << 40) + 2), MIS),
    (dict(starts=1 << 40, lengths=(1 << 40) + 16), INV),       # outputs overlap
    (dict(starts=1 << 40, cached=(1 << 40) + 16), INV),        # an output overlaps an input
])
def test_tables_refusals(kw, code):
    assert bsm.lib().bsm_paged_tables(ctypes.addressof(_tables(**kw)), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n_tokens=-1), INV), (dict(n_heads=0), INV), (dict(head_dim=0), INV), (dict(page_size=0), INV),
    (dict(n_pages=0), INV), (dict(dtype=9), INV), (dict(k=None), INV), (dict(slots=None), INV),
    (dict(k_stride_token=64), INV),                             # tokens overlap
    (dict(kv_stride_page=1024), INV), (dict(kv_stride_head=-64), INV), (dict(kv_stride_page=1 << 60), INV),
    (dict(n_tokens=1, k_stride_token=3, k=(1 << 40) + 8), MIS),
    (dict(head_dim=60), MIS), (dict(k=(1 << 40) + 8), MIS), (dict(kv_stride_page=2052), MIS),
    (dict(n_heads=1 << 20, head_dim=1 << 12), UNS),
    (dict(k=1 << 40, k_cache=(1 << 40) + 256), INV), (dict(k_cache=1 << 40, v_cache=1 << 40), INV),
    (dict(n_tokens=0, k=None), bsm.OK),
])
def test_write_refusals(kw, code):
    assert bsm.lib().bsm_paged_write(ctypes.addressof(_write(**kw)), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n_requests=-1), INV), (dict(n_tokens=-1), INV), (dict(page_size=0), INV), (dict(table_width=0), INV),
    (dict(table_stride=4), INV), (dict(max_new=-1), INV), (dict(window=-1), INV), (dict(flags=2), INV),
    (dict(dtype=7), INV), (dict(scale=0.0), INV), (dict(scale=-1.0), INV), (dict(scale=float("nan")), INV),
    (dict(scale=float("inf")), INV), (dict(flags=0, window=5), INV), (dict(heads_q=5), INV), (dict(heads_kv=0), INV),
    (dict(heads_q=1), INV), (dict(head_dim=0), INV),
    (dict(dtype=bsm.F32), UNS), (dict(head_dim=60), UNS), (dict(head_dim=136, q_stride_head=136, q_stride_token=544), UNS),
    (dict(q=None), INV), (dict(out=None), INV), (dict(workspace=None), INV), (dict(tables=None), INV),
    (dict(n_pages=0), INV), (dict(q_stride_head=32), INV), (dict(out_stride_token=0), INV),
    (dict(kv_stride_page=64), INV),
    (dict(q=(1 << 40) + 8), MIS), (dict(out_stride_token=260), MIS), (dict(workspace=(1 << 40) + 16), MIS),
    (dict(lse=(1 << 40) + 2), MIS), (dict(q=1 << 40, out=1 << 40), INV), (dict(lse=1 << 40, out=1 << 40), INV),
    (dict(workspace=1 << 40, k_cache=(1 << 40) + (1 << 20)), INV),
    (dict(n_requests=0, q=None), bsm.OK), (dict(n_tokens=0, q=None), bsm.OK),
])
def test_attention_refusals(kw, code):
    assert bsm.lib().bsm_paged_attention(ctypes.addressof(_attention(**kw)), None) == code


def test_null_descriptors_and_bad_workspace_arguments():
    assert bsm.lib().bsm_paged_tables(None, None) == INV
    assert bsm.lib().bsm_paged_write(None, None) == INV
    assert bsm.lib().bsm_paged_attention(None, None) == INV
    for args in [(5, 2, 64, 1), (4, 0, 64, 1), (4, 2, 65, 1), (4, 2, 192, 1), (4, 2, 64, -1)]:
        assert bsm.lib().bsm_paged_workspace_bytes(-1, *args) == -1
        with pytest.raises(ValueError):
            bsm.bsm_paged_workspace_bytes(*args)


def test_softmax_and_product_still_refuse_f16():
    L = bsm.lib()
    assert L.bsm_softmax(1 << 32, 1 << 33, 1, 4, 64, bsm.F16, bsm.POLICY_DYNAMIC, None) == INV
    assert L.bsm_bmm(1 << 32, 1 << 33, 1 << 34, 1, 128, 64, 64, bsm.F16, bsm.POLICY_DYNAMIC, None) == INV


def test_binding_refuses_tensors_the_library_cannot_see():
    import torch
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    with pytest.raises(ValueError):     # not on a GPU
        bsm.bsm_paged_write(z(3, 2, 64), z(3, 2, 64), z(4, 16, 2, 64), z(4, 16, 2, 64), z(3, dt=torch.int64))
    with pytest.raises(ValueError):     # types differ
        bsm.bsm_paged_write(z(3, 2, 64), z(3, 2, 64, dt=torch.float16), z(4, 16, 2, 64), z(4, 16, 2, 64),
                            z(3, dt=torch.int64))


def test_descriptors_match_the_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    pairs = [("bsm_paged_tables_desc", bsm.PagedTablesDesc), ("bsm_paged_write_desc", bsm.PagedWriteDesc),
             ("bsm_paged_desc", bsm.PagedDesc)]
    body = "".join('  printf("%%zu\\n", sizeof(%s));\n' % c for c, _ in pairs)
    body += "".join('  printf("%%zu\\n", offsetof(%s, %s));\n' % (c, f[0]) for c, p in pairs for f in p._fields_)
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "bsm.h"\nint main(void) {\n%s  return 0;\n}\n' % body)
    exe = tmp_path / "s"
    subprocess.run([gcc, "-I", os.path.dirname(bsm.HEADER), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = [ctypes.sizeof(p) for _, p in pairs] + [getattr(p, f[0]).offset for _, p in pairs for f in p._fields_]
    assert got == want
