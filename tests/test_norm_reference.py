"""The 64-bit reference of the norm's tests against torch.autograd and against differences (CPU)."""
import pytest
import torch

import norm_util


def plain(X, offsets, groups, w, b, eps, act):
    parts = []
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        if hi == lo:
            continue
        x = X[lo:hi].reshape(hi - lo, groups, -1)
        mean = x.mean((0, 2), keepdim=True)
        x = (x - mean) / torch.sqrt(((x - mean) ** 2).mean((0, 2), keepdim=True) + eps)
        z = x.reshape(hi - lo, -1) * w + b
        parts.append(torch.relu(z) if act == "relu" else torch.nn.functional.silu(z) if act == "silu" else z)
    return torch.cat(parts)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("groups", [1, 3, 12])
def test_reference(act, groups):
    torch.manual_seed(groups)
    offsets = [0, 5, 5, 6, 20]
    X, dY = (torch.randn(20, 12, dtype=torch.float64) for _ in range(2))
    w, b = torch.randn(12, dtype=torch.float64), torch.randn(12, dtype=torch.float64)
    leaves = [t.clone().requires_grad_() for t in (X, w, b)]
    want = plain(leaves[0], offsets, groups, *leaves[1:], 1e-5, act)
    y, stats, _, _ = norm_util.forward(X, offsets, groups, w, b, 1e-5, act)
    assert torch.allclose(y, want, rtol=1e-12, atol=1e-12)
    got, _ = norm_util.backward(dY, X, offsets, groups, w, b, stats, act)
    for g, t in zip(got, torch.autograd.grad((want * dY).sum(), leaves)):
        assert torch.allclose(g, t, rtol=1e-9, atol=1e-9)
    f = lambda X: float((plain(X, offsets, groups, w, b, 1e-5, act) * dY).sum())  # noqa: E731
    for i, j in ((0, 0), (3, 7), (12, 11)):
        e = torch.zeros_like(X)
        e[i, j] = 1e-6
        assert abs((f(X + e) - f(X - e)) / 2e-6 - float(got[0][i, j])) <= 1e-6 * (1 + abs(float(got[0][i, j])))
