"""SiLU of the group norm far from zero on both sides: its derivative is 1 above, whatever the size of z, and results and gradients have
fp32's relative accuracy."""
import pytest
import torch

import norm_util
from test_gpu_norm import ACTS, BF16, DEV, F32, empty_graph

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# a cluster, short graphs, pieces of rows, one block for a group
KINDS = {"a cluster": (640, None), "a batch": (4000, "batch"), "pieces": (40000, None), "no scratch": (40000, "no scratch")}


def sigmoid_error(z):
    """Relative error of s = 1 / (1 + t) and of t = exp(-z), in units of 2^-24: the exponent z log2 e is off by two roundings (ln 2 of
    that: 1.5 |z| covers it), 2^x by 2^-22; 1 + t is rounded, and 1 / is that of a product of two: two more roundings and 2^-23."""
    t = 4 + 1.5 * z.abs()
    return t, torch.sigmoid(-z) * t + 5


def setup(n, how, x_type, y_type, F, size, seed):
    g = empty_graph(n)
    offsets = [0, n]
    if how == "batch":
        offsets = sorted([0, *range(7, n, 13), n])
        g.dg_graph_set_batch(offsets)
    elif how == "no scratch":
        g.dg_graph_set_param("scratch_mb", 0)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=DEV, generator=gen)  # noqa: E731
    X, dY = r(n, F).to(x_type), (0.1 * r(n, F)).to(y_type)
    # statistics that round nothing: hat is x itself
    stats = torch.tensor([0.0, 1.0], device=DEV).expand(len(offsets) - 1, 2, 2).contiguous()
    w = (1 + 0.1 * r(F)).abs()
    # every other channel, and a few neighbours, far from zero: what a kernel shares between channels has to serve both
    far = torch.arange(F, device=DEV) % 4 != 1
    return g, offsets, X, dY, stats, w, torch.where(far, size * (1 + 0.1 * r(F).abs()), r(F))


@pytest.mark.parametrize("size", [0.0, 3.0, 10.0, 17.0, 30.0, 100.0, 1e4, 1e6, 1e8, 1e20, -3.0, -10.0, -30.0, -41.0, -60.0, -1e6, -1e20])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("x_type,y_type", [(F32, F32), (BF16, BF16), (F32, BF16)])
def test_gradients_of_silu_far_from_zero(x_type, y_type, kind, size):
    n, how = KINDS[kind]
    F, groups = 16, 2
    g, offsets, X, dY, stats, w, b = setup(n, how, x_type, y_type, F, size, 3)
    got = g.dg_group_norm_bwd(dY, X, stats, groups, w, b, ACTS["silu"])

    x, dy, w64, b64 = X.double(), dY.double(), w.double(), b.double()
    z = x * w64 + b64                     # in fp32: one rounding
    t = torch.exp(-z.clamp(min=-60))
    s = 1 / (1 + t)
    far = z < -43                         # taken for -43 there: s (1 + z (1 - s)) is below 1e-17
    v = torch.where(far, 0.0, z * t * s)  # z (1 - s)
    s = torch.where(far, 0.0, s)
    d = dy * s * (1 + v)
    # v: t's error times s (1 - s hangs on t so much), three roundings more; 1 + v, the two products; z's own rounding times the
    # second derivative, 1/2 at most and below (2 + |z|) exp(-|z|)
    of_t, of_s = sigmoid_error(z.clamp(-43, 43))
    of_v = v.abs() * (s * of_t + 5 + 3)
    second = torch.minimum(torch.full_like(z, 0.5), (2 + z.abs()) * torch.exp(-z.abs()))
    d_d = U * dy.abs() * (s * (of_v + (1 + v).abs()) + (s * (1 + v)).abs() * (of_s + 2) + second * z.abs()) + 1e-16 * dy.abs()
    row = norm_util.rows_of(offsets).to(DEV)
    q, width, rows = d * w64, F // groups, norm_util.CHAIN
    d_q = d_d * w64 + U * q.abs()
    mean = lambda v: norm_util.spread(norm_util.mean_over(v, row, offsets, groups), row, width)  # noqa: E731
    dX = q - mean(q) - x * mean(q * x)
    d_A = mean(d_q) + rows * U * mean(q.abs())
    d_B = mean(d_q * x.abs()) + (rows + 1) * U * mean((q * x).abs())
    d_dX = d_q + d_A + x.abs() * d_B + 4 * U * (q.abs() + mean(q).abs() + (x * mean(q * x)).abs())
    dw, db = (d * x).sum(0), d.sum(0)
    d_dw = (d_d * x.abs()).sum(0) + (rows + 1) * U * (d * x).abs().sum(0)
    d_db = d_d.sum(0) + rows * U * d.abs().sum(0)
    for name, a, want, bound, dtype in (("dX", got[0], dX, d_dX, x_type), ("dw", got[1], dw, d_dw, F32), ("db", got[2], db, d_db, F32)):
        off, most = (a.double() - want).abs(), norm_util.rounded(want, bound, dtype)
        assert bool((off <= most).all()), (name, float((off / most).max()))


@pytest.mark.parametrize("size", [0.0, 10.0, 100.0, 1e6, 1e20, -10.0, -41.0, -60.0, -1e20])
@pytest.mark.parametrize("kind", list(KINDS))
def test_silu_far_from_zero(kind, size):
    n, how = KINDS[kind]
    F, groups = 16, 2
    g, offsets, X, _, _, w, b = setup(n, how, F32, F32, F, size, 4)
    Y, stats = g.dg_group_norm_fwd(X, groups, w, b, act=ACTS["silu"])
    row = norm_util.rows_of(offsets).to(DEV)
    mean, rstd = (norm_util.spread(stats[..., k].double(), row, F // groups) for k in (0, 1))
    hat = (X.double() - mean) * rstd
    z = hat * w.double() + b.double()
    y = torch.where(z < -60, 0.0, z / (1 + torch.exp(-z.clamp(min=-60))))
    # hat: two roundings; z: one of the sum; s, and the product
    d_z = U * (2.01 * (hat * w.double()).abs() + z.abs())
    _, of_s = sigmoid_error(z.clamp(-43, 43))
    assert bool(((Y.double() - y).abs() <= 1.1 * d_z * torch.sigmoid(z + 3).clamp(min=0) + U * y.abs() * (of_s + 1) + 1e-16).all())
