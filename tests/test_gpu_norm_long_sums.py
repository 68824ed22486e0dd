"""Group norm over graphs of which a thread has thousands of rows: statistics with rows far from the others in front of them, and
sums whose roundings all go one way, against 64 bits.  No sum in 32 bits goes over more than 64 rows."""
import pytest
import torch

import norm_util
from test_gpu_norm import BF16, DEV, F32, empty_graph

pytestmark = pytest.mark.gpu
U = norm_util.U


def long_matrix(n, F, dtype, front, seed):
    """Numbers about 0.7 with a spread of 1 and, in the first rows, numbers far away."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    X = torch.empty(n, F, dtype=dtype, device=DEV)
    for lo in range(0, n, 250_000):
        X[lo:lo + 250_000] = torch.randn(min(250_000, n - lo), F, device=DEV, generator=gen) + 0.7
    X[:len(front)] += torch.tensor(front, device=DEV).to(dtype).view(-1, 1)
    return X


def moments(X, groups):
    """(mean, variance, mean of |x|) of every group in 64 bits."""
    n, F = X.shape
    part = lambda lo: X[lo:lo + 100_000].double().view(-1, groups, F // groups)  # noqa: E731
    cells = n * (F // groups)
    mean = sum(part(lo).sum((0, 2)) for lo in range(0, n, 100_000)) / cells
    var = sum((part(lo) - mean.view(1, -1, 1)).square().sum((0, 2)) for lo in range(0, n, 100_000)) / cells
    size = sum(part(lo).abs().sum((0, 2)) for lo in range(0, n, 100_000)) / cells
    return mean, var, size


FRONTS = {"one row": lambda far: [far], "hubs first": lambda far: [far / (i + 1) for i in range(1000)]}


@pytest.mark.parametrize("front", list(FRONTS))
@pytest.mark.parametrize("far", [1e3, 1e4])
@pytest.mark.parametrize("n,F,groups,dtype", [(1_000_000, 1024, 1024, F32), (1_000_000, 1024, 8, F32), (4_000_000, 255, 255, F32),
                                              (4_000_000, 512, 512, BF16), (4_000_000, 254, 2, BF16)])
def test_statistics_with_far_rows_in_front(n, F, groups, dtype, far, front):
    X = long_matrix(n, F, dtype, FRONTS[front](far), F)
    mean, var, size = moments(X, groups)
    _, stats = empty_graph(n).dg_group_norm_fwd(X, groups)
    # norm_util's: 64 rows and the joins behind them, relative to the sums of |x| and of squares about the mean of the 64 rows before,
    # which are at most twice the squares about the thread's mean
    d_mean = (norm_util.CHAIN + 1) * U * size
    d_var = 2 * (norm_util.CHAIN + 3) * U * var + d_mean.square()
    rstd = 1 / torch.sqrt(var + 1e-5)
    assert bool(((stats[0, :, 0].double() - mean).abs() <= d_mean).all())
    off = ((stats[0, :, 1].double() / rstd - 1).abs() / (d_var / var / 2 * 1.01 + U)).max()
    assert float(off) <= 1, float(off)


@pytest.mark.parametrize("n,F,groups,x_type,y_type", [(4_000_000, 255, 255, F32, F32), (4_000_000, 512, 8, BF16, BF16),
                                                      (4_000_000, 128, 8, F32, BF16), (4_000_000, 512, 512, BF16, F32)])
def test_sums_whose_roundings_go_one_way(n, F, groups, x_type, y_type):
    # numbers that lose the same bits at every addition to a large sum
    x, dy = (float(torch.tensor(v, dtype=t)) for v, t in ((1 + 0.4 * 2.0 ** -6, x_type), (1 + 0.3 * 2.0 ** -6, y_type)))
    X, dY = torch.full((n, F), x, dtype=x_type, device=DEV), torch.full((n, F), dy, dtype=y_type, device=DEV)
    stats = torch.tensor([0.0, 1.0], device=DEV).expand(1, groups, 2).contiguous()
    dX, dweight, dbias = empty_graph(n).dg_group_norm_bwd(dY, X, stats, groups)
    # 4 rows are added, then 16 of those sums; the rest is in 64 bits and rounded twice
    most = (4 + 16 + 2) * U
    assert float((dbias.double() / (n * dy) - 1).abs().max()) <= most
    assert float((dweight.double() / (n * dy * x) - 1).abs().max()) <= most + U       # the product is rounded too
    # A = dy, B = dy x, rounded once more; dX = dy - A - x B by three operations
    want = dy - dy - x * (dy * x)
    assert float((dX.double() - want).abs().max()) <= (most + 4 * U) * (dy + dy * x * x) + norm_util.HALF_STEP[x_type] * abs(want)
