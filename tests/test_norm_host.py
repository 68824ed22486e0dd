"""What the group norm refuses, and its host side, without a GPU."""
import ctypes

import pytest
import torch

from paper_2104_06700_b200 import binding
from test_host_side import fake, library  # noqa: F401

i64, f32 = ctypes.c_int64, ctypes.c_float


def batch(fake, g, *offsets):
    return fake.lib.dg_graph_set_batch(g, i64(len(offsets) - 1), (i64 * len(offsets))(*offsets))


def test_batches_that_are_refused(fake):
    g = fake.graph(64, 256)
    bad = binding.DG_ERR_INVALID_ARG
    assert batch(fake, g, 0, 10, 64) == binding.DG_OK
    assert batch(fake, g, 1, 10, 64) == bad
    assert batch(fake, g, 0, 10, 9) == bad
    assert batch(fake, g, 0, 65) == bad
    assert batch(fake, g, 0, -1, 3) == bad
    assert fake.lib.dg_graph_set_batch(g, i64(-1), None) == bad
    assert fake.lib.dg_graph_set_batch(g, i64(2), None) == bad
    assert fake.lib.dg_graph_set_batch(None, i64(0), None) == bad
    fake.lib.fake_alloc_limit(0)
    assert batch(fake, g, 0, 64) == binding.DG_ERR_CUDA
    fake.lib.fake_alloc_limit(ctypes.c_size_t(-1).value)
    assert fake.lib.dg_graph_set_batch(g, i64(0), None) == binding.DG_OK
    fake.lib.dg_graph_destroy(g)


def calls(fake, g, F=12, groups=4, x_type=0, y_type=0, act=1, eps=1e-5, **moved):
    n = 64
    p = {k: fake.array(n, F) for k in ("X", "Y", "dY", "dX")}
    p.update(dweight=fake.array(F), dbias=fake.array(F))
    p.update(weight=fake.array(F), bias=fake.array(F), stats=ctypes.c_void_p((fake.array(4 * F).value + 7) // 8 * 8))
    p.update(moved)
    fwd = fake.lib.dg_group_norm_fwd(g, p["X"], x_type, F, groups, p["weight"], p["bias"], f32(eps), act, p["Y"], y_type,
                                     p["stats"], None)
    bwd = fake.lib.dg_group_norm_bwd(g, p["dY"], y_type, p["X"], x_type, F, groups, p["weight"], p["bias"], p["stats"], act,
                                     p["dX"], p["dweight"], p["dbias"], None)
    return fwd, bwd


def test_arguments_that_are_refused(fake):
    g = fake.graph(64, 256)
    ok, bad = binding.DG_OK, binding.DG_ERR_INVALID_ARG
    assert calls(fake, g) == (ok, ok)
    for wrong in (dict(F=0), dict(F=(1 << 20) + 1), dict(groups=0), dict(groups=5), dict(groups=24), dict(groups=-4),
                  dict(x_type=2), dict(y_type=-1), dict(act=3), dict(act=-1), dict(X=None), dict(stats=None)):
        assert calls(fake, g, **wrong) == (bad, bad), wrong
    for eps in (-1e-5, float("nan")):
        assert calls(fake, g, eps=eps) == (bad, ok)
    assert calls(fake, g, Y=None) == (bad, ok) and calls(fake, g, dY=None) == (ok, bad)
    assert calls(fake, g, dX=None, weight=None, bias=None) == (ok, ok)
    X = fake.array(2 * 64, 12)
    inside = ctypes.c_void_p(X.value + 64 * 12 * 4 - 4)
    assert calls(fake, g, X=X, Y=inside, dX=inside) == (bad, bad)
    assert calls(fake, g, X=X, Y=X, dX=X) == (bad, bad)
    dY = fake.array(64, 12)
    assert calls(fake, g, dY=dY, dX=dY) == (ok, bad)
    stats = ctypes.c_void_p((fake.array(60).value + 7) // 8 * 8 + 4)
    assert calls(fake, g, stats=stats) == (bad, bad)
    for name in ("X", "Y", "dY", "dX"):
        odd = ctypes.c_void_p(fake.array(65, 12).value + 2)
        got = calls(fake, g, **{name: odd})
        assert got == ((bad if name in "XY" else ok), (ok if name == "Y" else bad)), name
    for name in ("weight", "bias", "dweight", "dbias"):
        odd = ctypes.c_void_p(fake.array(20).value + 2)
        assert calls(fake, g, **{name: odd}) == (ok if name[0] == "d" else bad, bad), name
    assert calls(fake, None) == (bad, bad)
    fake.lib.dg_graph_destroy(g)


def test_more_statistics_than_blocks_are_refused(fake):
    g = fake.graph(64, 256)
    many = (i64 * 4098)(*([0] * 4097), 64)
    assert fake.lib.dg_graph_set_batch(g, i64(4097), many) == binding.DG_OK
    F = 1 << 19
    p = ctypes.c_void_p(1 << 40)        # not read: the call is refused first
    got = fake.lib.dg_group_norm_fwd(g, p, 0, F, F, None, None, f32(0.0), 0, ctypes.c_void_p(1 << 44), 0, p, None)
    assert got == binding.DG_ERR_UNSUPPORTED
    fake.lib.dg_graph_destroy(g)


@pytest.mark.parametrize("how", ["no memory", "scratch_mb"])
def test_the_norm_does_without_scratch(fake, how):
    g = fake.graph(64, 256)
    fake.events()
    if how == "no memory":
        fake.lib.fake_alloc_limit(0)
    else:
        assert fake.lib.dg_graph_set_param(g, b"scratch_mb", i64(0)) == binding.DG_OK
    assert calls(fake, g) == (binding.DG_OK, binding.DG_OK)
    names = [what for what, _, _ in fake.events()]
    assert "alloc" not in names and any("norm" in what for what in names)
    fake.lib.dg_graph_destroy(g)


def test_a_launch_that_fails_is_an_error(fake):
    g = fake.graph(64, 256)
    fake.lib.fake_failing_kernel(b"norm_")
    assert calls(fake, g) == (binding.DG_ERR_CUDA, binding.DG_ERR_CUDA)
    fake.lib.dg_graph_destroy(g)


def test_the_binding_checks_shapes_and_types():
    g = binding.Graph.__new__(binding.Graph)
    g.n, g._h, g.batch = 6, None, None
    X, w = torch.zeros(6, 8), torch.zeros(8)
    stats = torch.zeros(1, 2, 2)
    for call in (lambda: g.dg_group_norm_fwd(X[:5], 2, w, w), lambda: g.dg_group_norm_fwd(X, 3, w, w),
                 lambda: g.dg_group_norm_fwd(X, 0, w, w), lambda: g.dg_group_norm_fwd(X, 2, w[1:], w),
                 lambda: g.dg_group_norm_fwd(X, 2, w, w[1:]), lambda: g.dg_group_norm_fwd(X, 2, w, w, Y=X[:, :4]),
                 lambda: g.dg_group_norm_fwd(X, 2, w, w, stats=stats[:, 1:]),
                 lambda: g.dg_group_norm_bwd(X[:5], X, stats, 2, w, w), lambda: g.dg_group_norm_bwd(X, X, stats[:, 1:], 2, w, w),
                 lambda: g.dg_group_norm_bwd(X, X, stats, 2, w, w, dX=X[:5]), lambda: g.dg_group_norm_fwd(X, 2, w, w),
                 lambda: g.dg_graph_set_batch([0]), lambda: g.dg_graph_set_batch([0.0, 6.0])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: g.dg_group_norm_fwd(X, 2, w, w, Y=X.clone(), y_dtype=torch.bfloat16),
                 lambda: g.dg_group_norm_bwd(X, X, stats, 2, w, w, dX=X.to(torch.bfloat16)),
                 lambda: g.dg_group_norm_fwd(X.half(), 2, w, w)):
        with pytest.raises(TypeError):
            call()
