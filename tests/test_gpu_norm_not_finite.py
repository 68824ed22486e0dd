"""Group norm with an activation: a number that is not finite stays in its group where neighbouring channels are two groups' (widths of one and of
odd numbers, so that a pair of channels lies in two)."""
import pytest
import torch

from test_gpu_norm import ACTS, BF16, DEV, F32, empty_graph, inputs

pytestmark = pytest.mark.gpu
KINDS = {"a cluster": (600, None), "a batch": (4000, "batch"), "pieces": (40000, None), "no scratch": (40000, "no scratch")}


def handle(n, how):
    g = empty_graph(n)
    offsets = [0, n]
    if how == "batch":
        offsets = sorted([0, 0, 1, n, *range(7, n, 13)])
        g.dg_graph_set_batch(offsets)
    elif how == "no scratch":
        g.dg_graph_set_param("scratch_mb", 0)
    return g, offsets


def same(a, b, but, near=None):
    """Every number that is not in `but` is the same, bit for bit or within `near`; those there are NaN."""
    assert bool(a[but].isnan().all()) and not bool(b.isnan().any())
    if near is None:
        assert torch.equal(a[~but], b[~but])
    else:
        assert bool(((a.double() - b.double()).abs() <= near)[~but].all())


def roundings(Y, dY, X, stats, w, act, row_graph, groups):
    """How far SiLU's results may move when a neighbouring channel changes: its kernels take one reciprocal for two channels, so
    the sigmoid's roundings (a product, a reciprocal to 2^-23, a product, all with both sides: 8 times 2^-24) hang on both."""
    if act != "silu":
        return [None] * 4
    u, half = 2.0 ** -24, 2.0 ** -7        # 2^-7: a bf16 result on the other side of a border between two
    step = lambda t: half * t.double().abs() if t.dtype == BF16 else 2 * u * t.double().abs()  # noqa: E731
    width = X.shape[1] // groups
    spread = lambda k: stats[..., k][row_graph].repeat_interleave(width, 1).double()  # noqa: E731
    hat = (X.double() - spread(0)) * spread(1)
    z = hat.abs() * w.double().abs() + 2           # biases are below 2
    d = 9 * u * (1 + z) * dY.double().abs()        # s (1 + z (1 - s)): s <= 1 is off by 8 u of itself
    y = Y.double().abs() * 8 * u + step(Y)
    db, dw = d.sum(0), (d * hat.abs()).sum(0)
    # the group's means of d w and of d w hat, each at most the largest of them
    q = (d * w.double().abs()).max()
    dX = spread(1) * q * (2 + hat.abs() * hat.abs().max()) * 2
    return [y, dX + (half if X.dtype == BF16 else 2 * u) * 20 * spread(1), dw + 2 * u * (dY.double().abs() * hat.abs()).sum(0),
            db + 2 * u * dY.double().abs().sum(0)]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("F,groups", [(8, 8), (6, 2), (100, 20), (16, 16), (41, 41)])
@pytest.mark.parametrize("x_type,y_type", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_a_group_keeps_what_is_not_finite(F, groups, x_type, y_type, kind, act):
    n, how = KINDS[kind]
    g, offsets = handle(n, how)
    X, dY, w, b = inputs(n, F, x_type, y_type, F)
    width = F // groups
    channel = width * (groups // 2) - 1           # the last of its group: its neighbour is another one's
    cells = torch.zeros(n, F, dtype=torch.bool, device=DEV)
    row = n // 2
    lo = max(o for o in offsets if o <= row)
    hi = min(o for o in offsets if o > row)
    graph, group = offsets.index(hi) - 1, channel // width
    cells[lo:hi, group * width:(group + 1) * width] = True
    of_group = torch.zeros(F, dtype=torch.bool, device=DEV)
    of_group[group * width:(group + 1) * width] = True
    only = torch.zeros(F, dtype=torch.bool, device=DEV)
    only[channel] = True

    def both_ways(X, dY, w, b, stats=None):
        Y, got = g.dg_group_norm_fwd(X, groups, w, b, act=ACTS[act], y_dtype=y_type)
        return (Y, got, *g.dg_group_norm_bwd(dY, X, got if stats is None else stats, groups, w, b, ACTS[act]))

    Y, stats, dX, dw, db = both_ways(X, dY, w, b)
    row_graph = torch.bucketize(torch.arange(n, device=DEV), torch.tensor(offsets, device=DEV), right=True) - 1
    of_y, of_dx, of_dw, of_db = roundings(Y, dY, X, stats, w, act, row_graph.clamp(max=len(offsets) - 2), groups)
    for bad in (float("nan"), float("inf"), float("-inf")):
        X2 = X.clone()
        X2[row, channel] = bad
        got = both_ways(X2, dY, w, b)
        same(got[0], Y, cells, of_y)
        at = torch.zeros_like(stats, dtype=torch.bool)
        at[graph, group] = True
        assert bool(got[1][graph, group].isnan().any())       # the mean may be an infinity
        assert torch.equal(got[1][~at], stats[~at])
        same(got[2], dX, cells, of_dx)
        same(got[3], dw, of_group, of_dw)
        if act == "silu":                         # (NaN is above the ReLU's border: its dY counts)
            same(got[4], db, of_group, of_db)
    # one cell of x that the statistics do not know of: its channel's sums, its group's means, no other group's
    X2 = X.clone()
    X2[row, channel] = float("nan")
    got = both_ways(X2, dY, w, b, stats)
    same(got[2], dX, cells, of_dx)
    same(got[3], dw, only, of_dw)
    # a weight or a bias: the column forward; its sums and its group backward
    column = only.expand(n, F)
    groups_column = of_group.expand(n, F)
    for which in range(2):
        wb = [w.clone(), b.clone()]
        wb[which][channel] = float("nan")
        got = both_ways(X, dY, *wb)
        same(got[0], Y, column, of_y)
        if act == "silu":
            same(got[3], dw, only, of_dw)
            same(got[4], db, only, of_db)
        if act == "silu" or which == 0:
            same(got[2], dX, groups_column, of_dx)
    # an upstream gradient
    dY2 = dY.clone()
    dY2[row, channel] = float("nan")
    if act == "silu":
        got = both_ways(X, dY2, w, b)
        same(got[2], dX, cells, of_dx)
        same(got[3], dw, only, of_dw)
        same(got[4], db, only, of_db)
