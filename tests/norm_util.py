"""Group norm with an activation in 64 bits, and how far the kernels' results may be from it."""
import torch

U = 2.0 ** -24                      # half a step of fp32, relative
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
# Roundings on the way of a number into a sum, at the sizes tested: a thread adds at most 8 rows of 8 channels in
# registers, 4 for each join of two parts of a thread (at most 16) and of a block's threads (at most 9 levels), and one at
# the end.
CHAIN = 8 * 8 + 4 * (16 + 9) + 1


def activation(z, act):
    return z.clamp(min=0) if act == "relu" else z / (1 + torch.exp(-z)) if act == "silu" else z


def derivative(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def rows_of(offsets):
    offsets = torch.as_tensor(offsets)
    return torch.repeat_interleave(torch.arange(offsets.numel() - 1), offsets[1:] - offsets[:-1])


def mean_over(v, row, offsets, groups):
    """(graphs, groups) means of an (rows, F) matrix"""
    graphs = len(offsets) - 1
    width = v.shape[1] // groups
    total = torch.zeros((graphs, groups), dtype=torch.float64, device=v.device)
    total.index_add_(0, row, v.view(-1, groups, width).sum(2))
    length = torch.as_tensor(offsets[1:]) - torch.as_tensor(offsets[:-1])
    return total / (length.clamp(min=1).double() * width).view(-1, 1).to(v.device)


def spread(stat, row, width):
    return stat[row].repeat_interleave(width, 1)


def forward(X, offsets, groups, weight, bias, eps, act):
    """Y and stats in 64 bits (the rows of the batch alone), and the bounds on the kernels' distance from them."""
    row = rows_of(offsets).to(X.device)
    x, width = X[:row.numel()].double(), X.shape[1] // groups
    w = torch.ones(X.shape[1], device=X.device).double() if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    mean = mean_over(x, row, offsets, groups)
    d = x - spread(mean, row, width)
    var = mean_over(d.square(), row, offsets, groups)
    rstd = 1 / torch.sqrt(var + eps)
    hat = d * spread(rstd, row, width)
    z = hat * w + b
    y = activation(z, act)
    # the mean: CHAIN roundings of numbers no larger than mean |x|; the variance: the same relative to itself (a square
    # is rounded twice more) and the square of the mean's error, joined parts' means being off by that
    d_mean = (CHAIN + 1) * U * mean_over(x.abs(), row, offsets, groups)
    d_var = 2 * (CHAIN + 3) * U * var + d_mean.square()
    d_rstd = rstd * (torch.where(var + eps > 0, d_var / (var + eps), 0.0) / 2 * 1.01 + U)
    # hat: a difference, a product; z: a product and a sum, rounded once or twice
    off = spread(rstd * d_mean, row, width) + hat.abs() * (spread(d_rstd / rstd, row, width) + 3 * U)
    dz = w.abs() * off + 2 * U * ((hat * w).abs() + b.abs())
    d_y = 1.1 * dz                       # no activation is steeper than 1.1
    if act == "silu":                    # the exponential, the sum, the quotient and the product
        d_y = d_y + y.abs() * U * 2 * (8 + 1.2 * z.abs())
    return y, torch.stack([mean, rstd], 2), d_y, torch.stack([d_mean, d_rstd], 2)


def rounded(y, bound, dtype):
    """The bound behind the rounding of a result to its type; numbers below the least normal one are off by its steps."""
    return bound + HALF_STEP[dtype] * (y.abs() + bound) + 2.0 ** -149


def backward(dY, X, offsets, groups, weight, bias, stats, act):
    """(dX, dweight, dbias) in 64 bits from the statistics given, and bounds."""
    row = rows_of(offsets).to(X.device)
    n, width = row.numel(), X.shape[1] // groups
    x, dy = X[:n].double(), dY[:n].double()
    w = torch.ones(X.shape[1], device=X.device).double() if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    mean, rstd = (spread(stats[..., k].double(), row, width) for k in (0, 1))
    hat = (x - mean) * rstd
    z = hat * w + b
    d = dy * derivative(z, act)
    q = d * w
    A, B = mean_over(q, row, offsets, groups), mean_over(q * hat, row, offsets, groups)
    a, bb = spread(A, row, width), spread(B, row, width)
    dX = rstd * (q - a - hat * bb)
    # d: z's error (three roundings) times the second derivative (at most 1/2), then the sigmoid and four products
    d_d = torch.zeros_like(d)
    if act == "silu":
        dz = 3 * U * ((hat * w).abs() + b.abs())
        d_d = dy.abs() * (0.5 * dz + U * 2 * (12 + 1.2 * z.abs()) * (1 + z.abs()) * torch.sigmoid(z))
    d_q = d_d * w.abs() + U * q.abs()
    d_hat = 2 * U * hat.abs()
    d_A = mean_over(d_q, row, offsets, groups) + CHAIN * U * mean_over(q.abs(), row, offsets, groups)
    d_B = (mean_over(d_q * hat.abs() + d_hat * q.abs(), row, offsets, groups)
           + (CHAIN + 1) * U * mean_over((q * hat).abs(), row, offsets, groups))
    d_dX = rstd.abs() * (d_q + spread(d_A, row, width) + hat.abs() * spread(d_B, row, width) + d_hat * bb.abs()
                         + 4 * U * (q.abs() + a.abs() + (hat * bb).abs()))
    dw, db = (d * hat).sum(0), d.sum(0)
    d_dw = (d_d * hat.abs() + d_hat * d.abs()).sum(0) + (CHAIN + 1) * U * (d * hat).abs().sum(0)
    d_db = d_d.sum(0) + CHAIN * U * d.abs().sum(0)
    return (dX, dw, db), (d_dX, d_dw, d_db)
