"""Norms, aggregation, products, loss, clipping and AdamW as a training epoch runs them, against the same epoch from torch's
operations in 64 bits; learned features; refusals of the model's and the epoch's options."""
import pytest
import torch

from paper_2104_06700_b200 import binding, graphsage, optim, synth
from parity_util import make_graph

pytestmark = pytest.mark.gpu
DEV = "cuda"


def union(sizes, seed):
    """A handle over the disjoint union of random graphs, its edges, and where each begins."""
    gen = torch.Generator().manual_seed(seed)
    offsets, src, dst = [0], [], []
    for n in sizes:
        if n:
            e = 6 * n
            src.append(torch.randint(0, n, (e,), generator=gen) + offsets[-1])
            dst.append(torch.randint(0, n, (e,), generator=gen) + offsets[-1])
        offsets.append(offsets[-1] + n)
    n = offsets[-1] + 9                    # padding behind the last graph
    src, dst = torch.cat(src), torch.cat(dst)
    rowptr, colidx, _ = synth._csr_from_edges(dst, src, n)
    g = binding.dg_graph_create(n, colidx.numel(), rowptr.to(DEV), colidx.to(DEV), None)
    g.dg_graph_transpose()
    return g, n, offsets, src.to(DEV), dst.to(DEV)


def reference_norm(Z, offsets, groups, w, b, eps, act):
    parts = []
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        if hi == lo:
            continue
        x = Z[lo:hi].reshape(hi - lo, groups, -1)
        mean = x.mean((0, 2), keepdim=True)
        x = (x - mean) / torch.sqrt(((x - mean) ** 2).mean((0, 2), keepdim=True) + eps)
        z = x.reshape(hi - lo, -1) * w + b
        parts.append(torch.nn.functional.silu(z) if act == "silu" else torch.relu(z))
    return torch.cat(parts + [torch.zeros_like(Z[offsets[-1]:])])


def reference_loss(X, params, src, dst, n, offsets, groups, act, labels, index, layers):
    deg1 = torch.bincount(dst, minlength=n).double() + 1
    H = X
    for i in range(layers):
        H = (torch.zeros_like(H).index_add_(0, dst, H[src]) + H) / deg1[:, None]
        H = H @ params[f"lin.{i}.weight"].t() + params[f"lin.{i}.bias"]
        if i + 1 < layers:
            H = reference_norm(H, offsets, groups, params[f"norms.{i}.weight"], params[f"norms.{i}.bias"], 1e-5, act)
    return torch.nn.functional.cross_entropy(H[index], labels[index])


@pytest.mark.parametrize("project_first", [False, True])
@pytest.mark.parametrize("act", ["relu", "silu"])
def test_an_epoch_matches_torch_in_64_bits(act, project_first):
    g, n, offsets, src, dst = union([40, 0, 1, 700, 260], 3)
    g.dg_graph_set_batch(offsets)
    dims = [24, 32, 16, 5]
    torch.manual_seed(1)
    model = graphsage.GraphSAGE(g, dims, project_first=project_first, norm_groups=4, activation=act).to(DEV)
    X = torch.nn.Parameter(torch.randn(n, 24, device=DEV))
    labels = torch.randint(0, 5, (n,), device=DEV)
    index = torch.arange(0, offsets[-1], 2, device=DEV)
    params = {k: p.detach().double().requires_grad_() for k, p in model.named_parameters()}
    X64 = X.detach().double().requires_grad_()
    other = torch.optim.AdamW([*params.values(), X64], lr=1e-2, weight_decay=5e-4)
    epoch = graphsage.make_epoch(model, X, labels, index, lr=1e-2, optimizer="adamw", max_norm=0.3)
    before = {k: p.detach().clone() for k, p in model.named_parameters()}
    loss = epoch()
    want = reference_loss(X64, params, src, dst, n, offsets, 4, act, labels, index, 3)
    want.backward()
    assert abs(float(loss) - float(want)) <= 1e-5 * abs(float(want))
    for k, p in [*model.named_parameters(), ("X", X)]:
        q = X64 if k == "X" else params[k]
        # products, aggregations and norms of a few thousand fp32 terms each: 2^-24 times some hundred of the largest one
        assert float((p.grad.double() - q.grad).abs().max()) <= 2e-5 * float(q.grad.abs().max()) + 1e-9, k
    # the norm of the gradients, and the step: from our gradients, so that only the step's own rounding is in question
    norm = torch.cat([p.grad.double().flatten() for p in [*model.parameters(), X]]).norm()
    assert abs(float(epoch.optimizer.grad_norm) - float(norm)) <= 1e-6 * float(norm)
    factor = min(1.0, 0.3 / (float(norm) + 1e-6))
    for k, p in model.named_parameters():
        gr = p.grad.double() * factor
        step = before[k].double() * (1 - 1e-2 * 5e-4) - 1e-2 * gr / (gr.abs() + 1e-8)   # the first step's quotient
        # m / sqrt(v): 12 roundings; where the gradient is near eps, its own rounding counts too
        assert float((p.detach().double() - step).abs().max()) <= 1e-2 * 1e-4 + 4 * 2.0 ** -24, k
    assert float(X.grad[offsets[-1]:].abs().max()) == 0        # padding learns nothing
    del other


@pytest.mark.parametrize("state_bits", [32, 8])
def test_epochs_with_bf16_rows_and_learned_features(state_bits):
    sg = synth.make("tiny", weighted=False)
    g = make_graph(sg)
    g.dg_graph_transpose()
    torch.manual_seed(2)
    dims = [64, 32, 32, 7]
    model = graphsage.GraphSAGE(g, dims, bf16_aggregate=True, norm_groups=8, activation="silu").to(DEV)
    X = torch.nn.Parameter(synth.features(sg.n, 64, 5, DEV).to(torch.bfloat16))
    labels = torch.randint(0, 7, (sg.n,), device=DEV)
    index = torch.arange(sg.n, device=DEV)
    epoch = graphsage.make_epoch(model, X, labels, index, optimizer="adamw", state_bits=state_bits, max_norm=1.0)
    with torch.no_grad():
        # the same model with fp32 rows: bf16 rounds each gathered number by 2^-9 of itself
        plain = graphsage.GraphSAGE(g, dims, norm_groups=8, activation="silu").to(DEV)
        plain.load_state_dict(model.state_dict())
        a, b = model(X), plain(X.float())
        assert a.dtype == torch.float32
        assert float((a - b).norm() / b.norm()) <= 0.05
    for _ in range(5):
        assert bool(epoch().isfinite())
    state = epoch.optimizer.state[X]
    assert torch.equal(X.detach(), state["master"].to(torch.bfloat16).view_as(X)) and int(state["step"]) == 5
    assert ("scales" in state) == (state_bits == 8)
    assert X.grad.dtype == torch.bfloat16 and bool(X.grad.isfinite().all())


def test_the_module_alone():
    g, n, offsets, _, _ = union([300, 5], 4)
    norm = graphsage.GroupNorm(g, 12, 3, "silu").to(DEV)
    X = torch.randn(12, n, device=DEV).t().requires_grad_()       # not contiguous
    g.dg_graph_set_batch(offsets)
    Y = norm(X)
    dY = torch.randn(n, 12, device=DEV)
    Y.backward(dY)
    X64 = X.detach().double().requires_grad_()
    w, b = (t.detach().double().requires_grad_() for t in (norm.weight, norm.bias))
    want = reference_norm(X64, offsets, 3, w, b, 1e-5, "silu")
    want.backward(dY.double())
    for a, c in ((Y, want), (X.grad, X64.grad), (norm.weight.grad, w.grad), (norm.bias.grad, b.grad)):
        assert float((a.detach().double() - c.detach()).abs().max()) <= 1e-5 * (1 + float(c.detach().abs().max()))
    assert norm(X.detach(), torch.bfloat16).dtype == torch.bfloat16
    free = graphsage.GroupNorm(g, 12, 3, "none", affine=False)
    assert list(free.parameters()) == [] and free(X.detach()).shape == (n, 12)
    Y = norm(X)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(Y.sum(), X, create_graph=True)[0].sum(), X)
    Y = norm(X)
    g.dg_graph_set_batch(None)
    with pytest.raises(RuntimeError, match="set_batch"):
        Y.sum().backward()


def test_options_that_are_refused():
    g, n, _, _, _ = union([30], 5)
    for wrong in (dict(norm_groups=5), dict(norm_groups=-1), dict(norm_groups=4, activation="gelu"), dict(activation="silu")):
        with pytest.raises(ValueError):
            graphsage.GraphSAGE(g, [8, 16, 4], **wrong)
    model = graphsage.GraphSAGE(g, [8, 16, 4], norm_groups=4).to(DEV)
    X, y, index = torch.randn(n, 8, device=DEV), torch.zeros(n, dtype=torch.int64, device=DEV), torch.arange(n, device=DEV)
    for wrong in (dict(optimizer="sgd"), dict(state_bits=8), dict(max_norm=1.0), dict(optimizer="adamw", state_bits=16)):
        with pytest.raises(ValueError):
            graphsage.make_epoch(model, X, y, index, **wrong)
    assert isinstance(graphsage.make_epoch(model, X, y, index).optimizer, torch.optim.Adam)
    assert isinstance(graphsage.make_epoch(model, X, y, index, optimizer="adamw").optimizer, optim.AdamW)
