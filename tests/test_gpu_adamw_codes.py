"""8-bit states of dg_adamw_step bit for bit: the formulas of dg.h operation by operation in numpy's fp32."""
import numpy as np
import pytest
import torch

import adamw_util as ref
from paper_2104_06700_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
F, ONE = np.float32, np.float32(1)


def codes_of(x, r16, root):
    """(codes without signs, scales) of numbers in blocks of 256."""
    blocks = np.pad(np.abs(x), (0, -x.size % 256)).reshape(-1, 256)
    scale = np.maximum(blocks.max(1) * (ONE / F(448)), F(2.0 ** -126))
    y = np.minimum(np.abs(x) * np.repeat(ONE / scale, 256)[:x.size], F(448))
    # steps of e4m3 at y: 2^-9 below 2^-6, then an eighth of the power of two; y + (r + 1/2) / 2^16 steps, rounded down
    y, r = y.astype(np.float64), (r16.astype(np.float64) + 0.5) / 2.0 ** 16
    y = np.where(y < 2.0 ** -6, (y.astype(F) + F(2.0 ** -6)).astype(np.float64) - 2.0 ** -6, y)   # at most 2^-30 off
    step = np.exp2(np.maximum(np.frexp(y)[1] - 4, -9).astype(np.float64))
    value = np.minimum((np.floor(y / step + r)) * step, 448.0)
    if root:
        value = np.where((x > 0) & (value == 0), 2.0 ** -9, value)
    return value, scale


@pytest.mark.parametrize("size", [1e-30, 1e-3, 1e10])
@pytest.mark.parametrize("n", [1, 255, 257, 4099, 300007])
def test_codes_and_scales_are_those_of_fp32_arithmetic(n, size):
    gen = torch.Generator(device=DEV).manual_seed(n)
    r = lambda: torch.randn(n, device=DEV, generator=gen)  # noqa: E731
    beta1, beta2, taken, seed = 0.9, 0.999, 12, 2 ** 35 + 5
    p, g = r(), r() * size * torch.exp(r())
    blocks = (n + 255) // 256
    scales = (torch.rand(blocks, 2, device=DEV, generator=gen) + 0.5) * size / 448
    m = (r() * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    u = (r().abs() * 100).clamp(max=448).to(torch.float8_e4m3fn)
    g[::5], m.view(torch.uint8)[::10], u.view(torch.uint8)[::10] = 0, 0, 0
    step = torch.tensor(taken, device=DEV)
    old = [t.float().cpu().numpy() for t in (m, u, g)]
    s = scales.cpu().numpy()
    lists = binding.AdamwList([g], [p], [m], [u], [step], [scales], ids=[3])
    binding.dg_adamw_step(lists, 1e-3, beta1, beta2, 1e-8, 0.0, binding.adamw_workspace(DEV), seed=seed)

    each = np.repeat(s, 256, 0)[:n]
    m0, u0, g0 = old[0] * each[:, 0], old[1] * each[:, 1], old[2]
    m1 = m0 + F(1 - beta1) * (g0 - m0)
    v1 = F(beta2) * (u0 * u0) + F(1 - beta2) * g0 * g0
    u1 = np.sqrt(v1)
    assert m1.dtype == u1.dtype == F
    bits = ref.random_bits(seed, taken, 3, 0, n, DEV).cpu().numpy()
    for got, x, r16, root, column in ((m, m1, bits & 0xFFFF, False, 0), (u, u1, bits >> 16, True, 1)):
        value, scale = codes_of(x, r16, root)
        assert np.array_equal(scales[:, column].cpu().numpy(), scale)
        assert np.array_equal(got.float().cpu().numpy().astype(np.float64), np.copysign(value, x))
