"""How the group norm shares out batches of graphs among blocks, without a GPU: whatever a kernel keeps in an array of fixed
length has to fit there."""
import ctypes
import os
import subprocess

import pytest

from paper_2104_06700_b200 import binding, build
from test_host_side import HERE, Fake

i64 = ctypes.c_int64
F32, BF16 = binding.DG_F32, binding.DG_BF16


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    build.build()
    objects = [os.path.join(build.BUILD_DIR, s[:-3] + ".o") for s in build.SOURCES]
    if not all(os.path.exists(o) for o in objects):  # the library came without them
        build.build(force=True)
    where = tmp_path_factory.mktemp("plans")
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-c", "-std=c++17", "-Xcompiler", "-fPIC", "-gencode",
                    "arch=compute_100a,code=sm_100a", "-I", build.INCLUDE, "-I", build.CSRC, "-o", str(where / "plans.o"),
                    os.path.join(HERE, "norm_plans.cu")], check=True)
    path = str(where / "libdgagg_plans.so")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", "-Wl,-Bsymbolic", "-I", cuda, "-o", path,
                    os.path.join(HERE, "fake_cudart.cpp"), str(where / "plans.o"), *objects], check=True)
    return Fake(path)


def plan(fake, g, F, groups, x_type, y_type, backward, rows_kept):
    out = (ctypes.c_longlong * 11)()
    fake.lib.norm_graph_plan(g, F, groups, x_type, y_type, int(backward), rows_kept, out)
    return out[:3], (out[3:7], out[7:11])


def widths():
    """(F, groups): instance norms, narrow groups of odd and even width, one group."""
    for F in (1, 2, 3, 7, 8, 41, 47, 64, 96, 100, 127, 128, 129, 136, 172, 192, 256, 300, 384, 500, 512, 602, 768, 1000, 1001, 1024,
              1030, 2048, 4096):
        for width in (1, 2, 3, 4, 5, 6, 7, 8, 9, 16, 24, 43, 64, 128, 250, 500, 512, F):
            if F % width == 0:
                yield F, F // width


@pytest.mark.parametrize("graphs,rows", [(1, 40), (1, 900), (7, 90), (300, 1), (300, 10), (1000, 64), (2048, 20), (2048, 64),
                                         (2048, 300), (9000, 3)])
def test_a_tile_holds_no_more_groups_than_its_arrays(plans, graphs, rows):
    n = graphs * rows
    g = plans.graph(n, 16)
    if graphs > 1:
        # sizes from none to several times the average
        cut = [min(n, (i * i * n) // (graphs * graphs)) for i in range(graphs)] + [n]
        assert plans.lib.dg_graph_set_batch(g, i64(graphs), (i64 * (graphs + 1))(*cut)) == binding.DG_OK
    most, threads = plans.lib.norm_tile_groups(), plans.lib.norm_graph_threads()
    taken = 0
    for F, groups in widths():
        for x_type, y_type in ((F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)):
            for backward, rows_kept in ((False, 12), (True, 8)):
                (blocks, long_blocks, cluster_log), shapes = plan(plans, g, F, groups, x_type, y_type, backward, rows_kept)
                if blocks == 0:
                    continue
                taken += 1
                assert 0 <= long_blocks <= blocks
                width = F // groups
                for vec, across, down, tiles in shapes[:1] if cluster_log else shapes:
                    what = (F, groups, x_type, y_type, backward, vec, across, down, tiles)
                    assert across * vec % width == 0, what                       # whole groups
                    assert across * vec // width <= most, what
                    assert 1 <= down and across * down <= threads, what
                    assert (tiles - 1) * across * vec < F <= tiles * across * vec, what
    assert taken
    plans.lib.dg_graph_destroy(g)
