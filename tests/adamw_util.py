"""One AdamW step in 64 bits, the hash its roundings go by, and the rounding rule."""
import math

import torch

U = 2.0 ** -24
LOW = 0xFFFFFFFF


def hash32(x):
    """lowbias32 on whole numbers (tensors of int64, or ints)"""
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        x = x ^ (x >> shift)
        x = (x * factor) & LOW
    return x ^ (x >> 16)


def random_bits(seed, taken, id, start, count, device):
    k = hash32((seed + 0x9E3779B9) & LOW)
    k = hash32(k ^ (seed >> 32 & LOW))
    k = hash32((k + taken) & LOW)
    key = hash32(k ^ id)
    at = torch.arange(start, start + count, device=device)
    high = at >> 32
    assert int(high.min()) == int(high.max())
    return hash32((at + hash32(key ^ int(high[0]))) & LOW)


def moments(g, m, v, factor, beta1, beta2):
    g = g.double() * factor
    return beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g


def new_param(p, m, v, t, lr, beta1, beta2, eps, decay):
    return p * (1 - lr * decay) - lr * (m / (1 - beta1 ** t)) / (torch.sqrt(v / (1 - beta2 ** t)) + eps)


def decoded(state, scales, which):
    """An 8-bit state as float64."""
    n = state.numel()
    return state.reshape(-1).float().double() * scales[:, which].double().repeat_interleave(256)[:n]


def scales_of(x):
    """Exact scales of |x| in blocks of 256, one for each number."""
    pad = torch.nn.functional.pad(x.abs(), (0, -x.numel() % 256)).view(-1, 256).amax(1)
    return (pad / 448).clamp(min=2.0 ** -126)


def rounded_8(x, r16):
    """(lower neighbour, step, how far from the next whole step the random bits bring |x|) in units of the scale; the
    result is lower + step where the third is >= 0."""
    scale = scales_of(x).repeat_interleave(256)[:x.numel()]
    y = (x.abs() / scale).clamp(max=448.0)
    step = torch.exp2(torch.frexp(y)[1].double() - 4).clamp(min=2.0 ** -9)
    q = y / step
    return torch.floor(q) * step * scale, step * scale, q - torch.floor(q) + (r16.double() * 16 + 8) / 2 ** 20 - 1


def check_8_bit(got, x, off, r16, root=False):
    """An 8-bit state `got` (float64) against x in 64 bits, which the kernel has with an error of `off`: the one of the two
    neighbours that the random bits choose, where rounding leaves no doubt, and one of them everywhere."""
    lower, step, over = rounded_8(x, r16)
    want = torch.where(over >= 0, lower + step, lower)
    scale = scales_of(x).repeat_interleave(256)[:x.numel()]
    if root:
        want = torch.where((x > 0) & (want == 0), 2.0 ** -9 * scale, want)
    want = torch.minimum(want, 448 * scale)
    # The scale is the block's largest number / 448 and inherits that number's error: relative to the scale at most the
    # largest `off` of the block over 448 scales (where m cancels, as 0.9 m + 0.1 g may, that is many roundings of m).  It
    # moves a number of at most 16 steps by 16 times that.  Beside it: the scale's quotient, its inverse, the product and
    # the shifted sum of small numbers, 8 roundings of at most 16 steps.
    scale_off = torch.nn.functional.pad(off, (0, -off.numel() % 256)).view(-1, 256).amax(1)
    scale_off = scale_off.repeat_interleave(256)[:x.numel()] / (448 * scale)
    doubt = off / step + 16 * (8 * U + scale_off) + 2.0 ** -19
    sure = (over.abs() > doubt) & (1 - over.abs() > doubt)
    near = (got.abs() - want).abs() <= (8 * U + scale_off) * want
    assert bool(near[sure].all()), int((~near[sure]).sum())
    assert int((~sure).sum()) <= 3 + 0.01 * x.numel()       # of the check itself: it leaves few numbers out
    assert bool(((got.abs() - x.abs()).abs() <= step * (1 + doubt) + (8 * U + scale_off) * x.abs()).all())
    if not root:
        assert bool(((got * x >= 0)).all())


def check_bf16(got, p, off, r16):
    """A randomly rounded bf16 parameter against p in 64 bits."""
    step = torch.exp2(torch.frexp(p)[1].double() - 8).clamp(min=2.0 ** -133)
    q = p.abs() / step
    over = q - torch.floor(q) + r16.double() / 2 ** 16 - 1
    want = p.sign() * (torch.floor(q) + (over >= 0)) * step
    doubt = off / step
    sure = (over.abs() > doubt) & (1 - over.abs() > doubt)
    assert torch.equal(got[sure], want[sure])
    assert int((~sure).sum()) <= 3 + 0.03 * p.numel()       # of the check itself: it leaves few numbers out
    assert bool(((got - p).abs() <= step * (1 + doubt)).all())


def close(x, want, bound):
    assert bool(((x.double() - want).abs() <= bound).all()), float(((x.double() - want).abs() - bound).max())


def isfinite(x):
    return math.isfinite(float(x))
