"""Which logits a selection reads: those of finished beams and of beams without a score
are not touched.  The logits lie in the host's memory, which this GPU reads through the
host's page tables; pages that nobody has touched are not there, and the kernel that
runs on the host's system says which are."""
import ctypes
import mmap

import numpy as np
import pytest
import torch

from oracle import beam_oracle as O
from paper_2002_07062_gb300 import bsm

pytestmark = pytest.mark.gpu
HOST_PAGE_TABLES = 100          # CUdevice_attribute: pageable memory through the host's page tables


class HostLogits:
    """fp32 rows in host memory of their own, each from the start of a page; nothing is touched yet."""

    def __init__(self, n, beams, vocab):
        self.n, self.beams, self.vocab = n, beams, vocab
        self.row = -(-vocab * 4 // mmap.PAGESIZE) * mmap.PAGESIZE
        self.map = mmap.mmap(-1, n * beams * self.row, flags=mmap.MAP_PRIVATE | mmap.MAP_ANONYMOUS)
        self.map.madvise(mmap.MADV_NOHUGEPAGE)
        self.values = np.frombuffer(self.map, np.float32).reshape(n, beams, self.row // 4)[:, :, :vocab]
        self.at = self.values.ctypes.data

    def touched(self):
        """[n, beams]: whether any page of the row is there."""
        pages = (ctypes.c_ubyte * (len(self.map) // mmap.PAGESIZE))()
        libc = ctypes.CDLL(None, use_errno=True)
        assert libc.mincore(ctypes.c_void_p(self.at), ctypes.c_size_t(len(self.map)), pages) == 0
        return (np.frombuffer(pages, np.uint8) & 1).reshape(self.n, self.beams, -1).any(2)


# (clusters, one and several lists a CTA; two launches; parts of several spans)
@pytest.mark.parametrize("n,beams,vocab", [(2, 4, 16000), (1, 20, 5000), (8, 3, 100), (20, 4, 16000), (1, 6, 100000)])
def test_logits_of_finished_and_unused_beams_are_not_touched(n, beams, vocab):
    v = ctypes.c_int()
    if ctypes.CDLL("libcuda.so.1").cuDeviceGetAttribute(ctypes.byref(v), HOST_PAGE_TABLES, 0) or not v.value:
        pytest.skip("the GPU does not read through the host's page tables")
    keep, rng = 6, np.random.default_rng(vocab)
    x = HostLogits(n, beams, vocab)
    scores = -rng.uniform(0, 3, (n, beams)).astype(np.float32)
    ended = np.zeros((n, beams), np.uint8)
    ended[:, 1] = 1                             # one finished beam a request, one that is not in use
    scores[:, 2] = [[-np.inf, np.nan, np.inf][r % 3] for r in range(n)]
    live = (ended == 0) & np.isfinite(scores)
    for r, b in zip(*live.nonzero()):
        x.values[r, b] = rng.standard_normal(vocab).astype(np.float32) * 3
    assert np.array_equal(x.touched(), live)
    s, e = torch.from_numpy(scores).cuda(), torch.from_numpy(ended).cuda()
    out, parents = torch.empty((n, keep), device="cuda"), torch.empty((n, keep), dtype=torch.int32, device="cuda")
    tokens = torch.empty_like(parents)
    ws = torch.empty(bsm.bsm_beam_select_workspace_bytes(n, beams, vocab, keep), dtype=torch.uint8, device="cuda")

    def run(finished):
        d = bsm.BeamSelectDesc(logits=x.at, scores=s.data_ptr(), ended=finished, out_scores=out.data_ptr(),
                               parents=parents.data_ptr(), tokens=tokens.data_ptr(), workspace=ws.data_ptr(),
                               workspace_bytes=ws.numel(), stride_request=beams * x.row // 4, stride_beam=x.row // 4,
                               n_requests=n, beams=beams, vocab=vocab, keep=keep, end_token=3, dtype=bsm.F32)
        assert bsm.lib().bsm_beam_select(ctypes.addressof(d), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()

    run(e.data_ptr())
    assert np.array_equal(x.touched(), live)
    val, par, tok = O.select(x.values, scores, keep, ended, 3)
    assert np.array_equal(parents.cpu().numpy(), par) and np.array_equal(tokens.cpu().numpy(), tok)
    assert np.abs(out.cpu().numpy() - val).max() < 1e-4
    # the same rows with nobody finished are read, and then they are there (and what the system brings beside them)
    run(None)
    assert x.touched()[np.isfinite(scores)].all()
