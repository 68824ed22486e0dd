"""Which way a layer of the model runs, without a GPU: what a layer's module does to its own hooks while it runs changes nothing behind
it."""
import types

import pytest
import torch

from paper_2104_06700_b200 import graphsage


def model_of(dims, **options):
    """A model whose aggregation is the identity, on the CPU."""
    graph = types.SimpleNamespace(rowptr=torch.zeros(7, dtype=torch.int64), n=6, dg_graph_get_param=lambda name: 0)
    model = graphsage.GraphSAGE(graph, dims, **options)
    model._aggregated = lambda M: M
    for lin in model.lin:
        lin.register_forward_hook(lambda *_: None)      # every layer calls its module
    return model


@pytest.mark.parametrize("project_first", [False, True])
def test_a_hook_that_removes_itself_keeps_the_relu(project_first):
    torch.manual_seed(0)
    model = model_of([4, 8, 5, 3], project_first=project_first)
    X = torch.randn(6, 4)
    want = model(X)
    H = X
    for i, lin in enumerate(model.lin):
        H = torch.nn.functional.linear(H, lin.weight, lin.bias)
        H = torch.relu(H) if i < 2 else H
    assert torch.allclose(want, H, atol=1e-6)
    assert bool((torch.nn.functional.linear(X, model.lin[0].weight, model.lin[0].bias) < 0).any())
    lin = model.lin[0]
    lin._forward_hooks.clear()
    calls = []

    def once(*_):
        calls.append(handle.remove())

    handle = lin.register_forward_hook(once)            # a lazy initialiser, a probe
    assert torch.equal(model(X), want) and len(calls) == 1 and graphsage._is_plain(lin)
