"""Group norm with an activation (dg_group_norm_fwd / _bwd) against the same formulas in 64 bits: types, groups of one channel
and of all, odd widths, batches of graphs with empty and one-row ones and with padding behind them, few and many rows."""
import pytest
import torch

import norm_util
from paper_2104_06700_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACTS = {"none": binding.DG_ACT_NONE, "relu": binding.DG_ACT_RELU, "silu": binding.DG_ACT_SILU}
F32, BF16 = torch.float32, torch.bfloat16


def empty_graph(n):
    return binding.dg_graph_create(n, 0, torch.zeros(n + 1, dtype=torch.int64, device=DEV),
                                   torch.zeros(0, dtype=torch.int32, device=DEV), None)


def ragged(n, graphs, behind, seed):
    """Offsets of `graphs` graphs: some empty, some of one row, one with a third of the rows."""
    gen = torch.Generator().manual_seed(seed)
    end = n - behind
    cut = torch.randint(0, end + 1, (graphs - 1,), generator=gen)
    if graphs > 5:
        cut[:3] = torch.tensor([0, end // 3, min(end, end // 3 + 1)])
        cut[3] = cut[4]
    return [0] + sorted(cut.tolist()) + [end]


def inputs(n, F, x_type, y_type, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=DEV, generator=gen)  # noqa: E731
    X = (r(n, F) * torch.exp(0.5 * r(F)) + 2 * r(F)).to(x_type)
    return X, (r(n, F) * 0.1).to(y_type), 1 + 0.3 * r(F), 0.3 * r(F)


def check(g, X, dY, groups, weight, bias, act, offsets, eps=1e-5):
    n, F = X.shape
    rows = offsets[-1]
    Y = torch.full((n, F), 7.0, device=DEV, dtype=dY.dtype)
    _, stats = g.dg_group_norm_fwd(X, groups, weight, bias, eps, ACTS[act], Y=Y)
    y, s, d_y, d_s = norm_util.forward(X, offsets, groups, weight, bias, eps, act)
    assert bool(((stats.double() - s).abs() <= d_s + 2.0 ** -149).all())
    assert bool(((Y[:rows].double() - y).abs() <= norm_util.rounded(y, d_y, Y.dtype)).all())
    assert bool((Y[rows:] == 7.0).all())

    given = s.float().contiguous()
    dX = torch.full_like(X, 7.0)
    got = g.dg_group_norm_bwd(dY, X, given, groups, weight, bias, ACTS[act], dX=dX)
    want, bounds = norm_util.backward(dY, X, offsets, groups, weight, bias, given, act)
    assert bool(((dX[:rows].double() - want[0]).abs() <= norm_util.rounded(want[0], bounds[0], X.dtype)).all())
    assert bool((dX[rows:] == 7.0).all())
    for a, b, bound in zip(got[1:], want[1:], bounds[1:]):
        assert bool(((a.double() - b).abs() <= norm_util.rounded(b, bound, F32)).all())
    return Y, stats, got


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("x_type,y_type", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("n,F,groups", [(1, 1, 1), (1, 8, 2), (2, 8, 8), (33, 47, 47), (257, 47, 1), (1000, 100, 20),
                                        (4096, 64, 8), (3001, 602, 14), (777, 256, 32)])
def test_one_graph(n, F, groups, x_type, y_type, act):
    g = empty_graph(n)
    check(g, *inputs(n, F, x_type, y_type, n + F)[:2], groups, *inputs(n, F, x_type, y_type, n + F)[2:], act, [0, n])


@pytest.mark.parametrize("n,F,groups,act", [(70001, 256, 32, "relu"), (30011, 47, 1, "silu"), (100003, 12, 3, "none"),
                                            (20001, 1028, 4, "silu"), (9001, 2050, 1, "relu"), (60000, 4, 4, "none"),
                                            (40961, 100, 100, "relu"), (6000, 2500, 1250, "silu")])
def test_many_rows(n, F, groups, act):
    for x_type, y_type in ((F32, F32), (BF16, BF16)):
        X, dY, w, b = inputs(n, F, x_type, y_type, n)
        check(empty_graph(n), X, dY, groups, w, b, act, [0, n])


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("n,F,groups,graphs,behind", [(500, 16, 4, 7, 0), (500, 47, 1, 40, 13), (5000, 128, 8, 300, 100),
                                                      (20000, 64, 64, 12, 1), (3, 8, 2, 9, 1), (64, 24, 3, 64, 64),
                                                      (40000, 40, 5, 6, 0), (9000, 300, 3, 2000, 7)])
def test_batches_of_graphs(n, F, groups, graphs, behind, act):
    offsets = ragged(n, graphs, behind, n + graphs)
    for x_type, y_type in ((F32, F32), (F32, BF16), (BF16, BF16)):
        X, dY, w, b = inputs(n, F, x_type, y_type, n)
        X[offsets[-1]:], dY[offsets[-1]:] = float("nan"), float("nan")   # padding is not read
        g = empty_graph(n)
        g.dg_graph_set_batch(offsets)
        check(g, X, dY, groups, w, b, act, offsets)


def test_without_weights_and_with_parts_of_the_gradients():
    n, F, groups = 3000, 36, 6
    X, dY, w, b = inputs(n, F, F32, F32, 1)
    g = empty_graph(n)
    check(g, X, dY, groups, None, None, "silu", [0, n])
    check(g, X, dY, groups, w, None, "relu", [0, n])
    check(g, X, dY, groups, None, b, "relu", [0, n])
    _, stats = g.dg_group_norm_fwd(X, groups, w, b)
    all_of_it = g.dg_group_norm_bwd(dY, X, stats, groups, w, b, ACTS["silu"])
    for k in range(3):
        want = {name: i == k for i, name in enumerate(("want_dX", "want_dweight", "want_dbias"))}
        part = g.dg_group_norm_bwd(dY, X, stats, groups, w, b, ACTS["silu"], **want)
        assert [p is not None for p in part] == [i == k for i in range(3)]
        assert torch.equal(part[k], all_of_it[k])


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_any_alignment(shift):
    n, F, groups = 2000, 64, 4
    for x_type, y_type in ((F32, F32), (BF16, BF16)):
        X, dY, w, b = inputs(n, F, x_type, y_type, shift)
        moved = [torch.empty(t.numel() + shift, dtype=t.dtype, device=DEV)[shift:].view(t.shape).copy_(t) for t in (X, dY, w, b)]
        check(empty_graph(n), moved[0], moved[1], groups, moved[2], moved[3], "silu", [0, n])


def test_large_means_and_small_spreads():
    """The variance is a mean of squares about the mean, not a difference of two large numbers."""
    n, F, groups = 50000, 32, 4
    X, dY, w, b = inputs(n, F, F32, F32, 2)
    check(empty_graph(n), X * 0.01 + 100, dY, groups, w, b, "none", [0, n])
    X[0] += 3e4      # one row far from the others
    check(empty_graph(n), X, dY, groups, w, b, "none", [0, n])
    X = torch.full((n, F), 3.0, device=DEV)   # no spread at all
    Y, stats = empty_graph(n).dg_group_norm_fwd(X, groups, w, b)
    assert torch.equal(Y, b.expand(n, F)) and bool((stats[..., 0] == 3.0).all())


def test_numbers_that_are_not_finite_stay_in_their_group():
    n, F, groups = 4000, 32, 4
    offsets = [0, 1500, 4000]
    X, dY, w, b = inputs(n, F, F32, F32, 3)
    g = empty_graph(n)
    g.dg_graph_set_batch(offsets)
    clean, _ = g.dg_group_norm_fwd(X, groups, w, b, act=ACTS["relu"])
    for bad in (float("nan"), float("inf")):
        X2 = X.clone()
        X2[10, 9] = bad                        # graph 0, group 1
        Y, stats = g.dg_group_norm_fwd(X2, groups, w, b, act=ACTS["relu"])
        assert bool(Y[:1500, 8:16].isnan().all()) and bool(stats[0, 1].isnan().any())
        rest = torch.ones(n, F, dtype=torch.bool, device=DEV)
        rest[:1500, 8:16] = False
        assert torch.equal(Y[rest], clean[rest])
    dY[2000, 0] = float("nan")
    _, stats = g.dg_group_norm_fwd(X, groups, w, b)
    dX, dw, db = g.dg_group_norm_bwd(dY, X, stats, groups, w, b)
    assert bool(dX[1500:, :8].isnan().all()) and not bool(dX[:1500].isnan().any()) and not bool(dX[:, 8:].isnan().any())
    assert dw.isnan().nonzero().flatten().tolist() == db.isnan().nonzero().flatten().tolist() == [0]


def test_the_gradient_of_relu_at_its_border():
    """Cells whose z is a rounding away from 0: the mask is the sign of z in 64 bits."""
    n, F = 4096, 64
    X, dY, w, b = inputs(n, F, F32, F32, 4)
    g = empty_graph(n)
    _, stats = g.dg_group_norm_fwd(X, 8, w, b)
    mean, rstd = (stats[0, :, k].repeat_interleave(8) for k in (0, 1))
    X = (mean - b / (w * rstd)).expand(n, F).contiguous()      # z = 0 up to rounding
    X = torch.where(torch.rand(n, F, device=DEV) < 0.5, torch.nextafter(X, X + 1), X)
    check_border = norm_util.backward(dY, X, [0, n], 8, w, b, stats, "relu")
    got = g.dg_group_norm_bwd(dY, X, stats, 8, w, b, ACTS["relu"])
    for a, want, bound in zip(got, *check_border):
        assert bool(((a.double() - want).abs() <= norm_util.rounded(want, bound, F32)).all())


@pytest.mark.parametrize("n,F,groups,graphs", [(5000, 128, 8, 1), (30000, 47, 47, 1), (3000, 100, 4, 50)])
def test_runs_repeat_and_scratch_is_not_needed(n, F, groups, graphs):
    X, dY, w, b = inputs(n, F, F32, BF16, n)
    offsets = ragged(n, graphs, 0, 5) if graphs > 1 else [0, n]
    g = empty_graph(n)
    if graphs > 1:
        g.dg_graph_set_batch(offsets)
    first = check(g, X, dY, groups, w, b, "silu", offsets)
    again = check(g, X, dY, groups, w, b, "silu", offsets)
    for a, c in zip((first[0], first[1], *first[2]), (again[0], again[1], *again[2])):
        assert torch.equal(a, c)
    g.dg_graph_set_param("scratch_mb", 0)
    check(g, X, dY, groups, w, b, "silu", offsets)


def test_streams_capture_and_a_changed_batch():
    n, F, groups = 6000, 64, 4
    X, dY, w, b = inputs(n, F, F32, F32, 6)
    g = empty_graph(n)
    want = g.dg_group_norm_fwd(X, groups, w, b, act=ACTS["silu"])
    want_back = g.dg_group_norm_bwd(dY, X, want[1], groups, w, b, ACTS["silu"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = g.dg_group_norm_fwd(X, groups, w, b, act=ACTS["silu"], stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

    static = X.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = g.dg_group_norm_fwd(static, groups, w, b, act=ACTS["silu"])
        back = g.dg_group_norm_bwd(dY, static, out[1], groups, w, b, ACTS["silu"])
    for _ in range(3):
        static.copy_(X * 2)
        graph.replay()
        static.copy_(X)
        graph.replay()
        for a, c in zip((*out, *back), (*want, *want_back)):
            assert torch.equal(a, c)
    del graph

    offsets = [0, 0, 100, 5900]
    g.dg_graph_set_batch(offsets)
    check(g, X, dY, groups, w, b, "relu", offsets)
    Y, _ = g.dg_group_norm_fwd(X, groups, w, b)
    assert bool((Y[5900:] == 0).all())       # a result that the call makes
    g.dg_graph_set_batch(torch.tensor(offsets, device=DEV))
    check(g, X, dY, groups, w, b, "relu", offsets)
    g.dg_graph_set_batch(None)
    assert torch.equal(g.dg_group_norm_fwd(X, groups, w, b, act=ACTS["silu"])[0], want[0])


def test_no_rows():
    g = empty_graph(0)
    X = torch.empty(0, 8, device=DEV)
    Y, stats = g.dg_group_norm_fwd(X, 2)
    assert Y.shape == (0, 8) and stats[0, :, 0].tolist() == [0.0, 0.0]
    assert torch.allclose(stats[..., 1], torch.full_like(stats[..., 1], 1e-5 ** -0.5))
    dX, dw, db = g.dg_group_norm_bwd(X, X, stats, 2)
    assert dX.shape == (0, 8) and not bool(dw.any()) and not bool(db.any())


def test_silu_far_below_zero():
    """Where exp(-z) leaves fp32: results and gradients vanish, whatever the size of z."""
    n, F = 3000, 8
    X, dY, w, b = inputs(n, F, F32, F32, 8)
    for big in (50.0, 1e3, 1e12, 1e30):
        for offsets in ([0, n], [0, 20, n]):        # one graph in pieces' kernels and in a cluster's, and a batch
            g = empty_graph(n)
            if len(offsets) > 2:
                g.dg_graph_set_batch(offsets)
            bias = b - big
            Y, stats = g.dg_group_norm_fwd(X, 2, w, bias, act=ACTS["silu"])
            y, _, _, _ = norm_util.forward(X, offsets, 2, w, bias, 1e-5, "silu")
            assert float((Y.double() - torch.nan_to_num(y)).abs().max()) <= 1e-12
            dX, dw, db = g.dg_group_norm_bwd(dY, X, stats, 2, w, bias, ACTS["silu"])
            assert all(float(t.abs().max()) <= 1e-10 for t in (dX, dw, db))
            bias = b + big
            Y, _ = g.dg_group_norm_fwd(X, 2, w, bias, act=ACTS["silu"])
            assert bool(((Y.double() - (b.double() + big)).abs() <= 1e-6 * big + 100).all())


def test_large_matrices_in_captured_graphs_and_two_streams():
    """The kernels of long graphs take scratch between their launches: a replay, an eager call and another stream's call at
    the same time do not share it."""
    n, F, groups = 70000, 64, 4
    X, dY, w, b = inputs(n, F, F32, BF16, 7)
    g = empty_graph(n)
    fwd = lambda X, **k: g.dg_group_norm_fwd(X, groups, w, b, act=ACTS["silu"], y_dtype=BF16, **k)  # noqa: E731
    want = [fwd(X * s) for s in (1, 3)]
    back = [g.dg_group_norm_bwd(dY, X * s, want[i][1], groups, w, b, ACTS["silu"]) for i, s in enumerate((1, 3))]
    static = [X.clone(), X * 3]
    graphs, outs = [], []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = fwd(static[i])
            outs.append((*y, *g.dg_group_norm_bwd(dY, static[i], y[1], groups, w, b, ACTS["silu"])))
        graphs.append(graph)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        eager = fwd(static[0])
        with torch.cuda.stream(side):
            other = fwd(static[1])
        torch.cuda.synchronize()
        for i, e in enumerate((eager, other)):
            for a, c in zip((*outs[i], *e), (*want[i], *back[i], *want[i])):
                assert torch.equal(a, c)
    del graphs


def test_more_cells_than_32_bits_count():
    n, F, groups = 9_000_000, 512, 8
    X = torch.empty(n, F, dtype=BF16, device=DEV)
    for lo in range(0, n, 1_000_000):
        X[lo:lo + 1_000_000].normal_(0.1 * (lo % 3), 1 + lo / n)
    dY = torch.empty_like(X).normal_(0, 0.1)
    _, _, w, b = inputs(4, F, F32, F32, 9)
    sums = torch.zeros(2, groups, dtype=torch.float64, device=DEV)
    for lo in range(0, n, 250_000):
        part = X[lo:lo + 250_000].double().view(-1, groups, F // groups)
        sums += torch.stack([part.sum((0, 2)), part.square().sum((0, 2))])
    mean = sums[0] / (n * (F // groups))
    rstd = (sums[1] / (n * (F // groups)) - mean.square() + 1e-5).rsqrt()
    for offsets in ([0, n], [0, 7, n - 2, n]):
        g = empty_graph(n)
        if len(offsets) > 2:
            g.dg_graph_set_batch(offsets)
        Y, stats = g.dg_group_norm_fwd(X, groups, w, b, act=ACTS["silu"])
        if len(offsets) == 2:
            # a thread adds some thousand rows: 2^-24 times their number at most, far less as roundings go both ways
            assert float((stats[0, :, 0].double() - mean).abs().max()) <= 1e-5
            assert float((stats[0, :, 1].double() / rstd - 1).abs().max()) <= 1e-5
        dX, dw, db = g.dg_group_norm_bwd(dY, X, stats, groups, w, b, ACTS["silu"])
        # the rows at both ends and about the places where 32-bit counts of cells end, from the statistics
        st = stats[-1 if len(offsets) == 2 else 1].double()
        for row in (10, 2 ** 31 // F - 3, 2 ** 32 // F - 3, n - 20):
            x, hi = X[row:row + 6].double(), row + 6
            hat = (x - st[:, 0].repeat_interleave(F // groups)) * st[:, 1].repeat_interleave(F // groups)
            z = hat * w.double() + b.double()
            y = z / (1 + torch.exp(-z))
            assert bool(((Y[row:hi].double() - y).abs() <= 2.0 ** -8 * y.abs() + 1e-4).all())
            s = torch.sigmoid(z)
            q = dY[row:hi].double() * (s * (1 + z * (1 - s))) * w.double()
            # A and B are means of nine million times 64 numbers of random sign: nearly nothing beside q
            want = q * st[:, 1].repeat_interleave(F // groups)
            assert bool(((dX[row:hi].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2e-3 * (1 + hat.abs())).all())
        del Y, dX
