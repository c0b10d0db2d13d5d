"""How a selection's rows are cut: through the library's own function, which the
public calls do not show."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2002_07062_gb300 import bsm

SOURCE = """
#include "bsm_beam.h"
#include "bsm_paged_host.h"
extern "C" int cut(int n, int beams, int vocab, int es, int n_sm, int clusters, int *out)
{
    const bsm::BeamCut c = bsm::beam_cut(n, beams, vocab, es, n_sm, clusters != 0);
    out[0] = c.parts;
    out[1] = c.part;
    return c.together;
}
extern "C" long long most_lists(long long rows, int n_sm) { return bsm::beam_most_lists(rows, n_sm); }
extern "C" int clusters_fit()
{
    bsm::PagedDev *d = nullptr;
    return bsm::paged_device(-1, &d) ? -1 : d->clusters;
}
"""


@pytest.fixture(scope="module")
def inner(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no C++ compiler")
    import __graft_entry__ as g
    g.build()
    at = tmp_path_factory.mktemp("cut")
    (at / "cut.cpp").write_text(SOURCE)
    lib_dir = os.path.dirname(bsm.LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(bsm.PKG, "csrc"), str(at / "cut.cpp"),
                    "-o", str(at / "cut.so"), bsm.LIB_PATH, "-Wl,-rpath," + lib_dir], check=True)
    bsm.lib()
    lib = ctypes.CDLL(str(at / "cut.so"))
    lib.most_lists.restype, lib.most_lists.argtypes = ctypes.c_longlong, [ctypes.c_longlong, ctypes.c_int]
    return lib


def _cut(lib, n, beams, vocab, es, n_sm, clusters):
    out = (ctypes.c_int * 2)()
    return bool(lib.cut(n, beams, vocab, es, n_sm, clusters, out)), out[0], out[1]


@pytest.mark.parametrize("n_sm", [152, 16, 4, 1])
@pytest.mark.parametrize("es", [2, 4])
def test_a_device_that_places_no_cluster_takes_two_launches(inner, n_sm, es):
    for n in (1, 2, 8, 9, 40):
        for beams in (1, 3, 16, 64):
            for vocab in (1, 7, 500, 5000, 32000, 128000, 1 << 20):
                together, parts, part = _cut(inner, n, beams, vocab, es, n_sm, 0)
                assert not together
                # all of a row, in whole pieces; lists that the workspace and the join have room for
                assert parts >= 1 and part % (16 // es) == 0 and (parts - 1) * part < vocab <= parts * part
                assert beams * parts <= 128 and n * beams * parts <= inner.most_lists(n * beams, n_sm)
                same = _cut(inner, n, beams, vocab, es, n_sm, 1)
                assert same[0] == (n <= 8 and beams * vocab * es <= 16 << 17)
                assert same[0] or same[1:] == (parts, part)


@pytest.mark.gpu
def test_this_device_places_them(inner):
    assert inner.clusters_fit() == 1
