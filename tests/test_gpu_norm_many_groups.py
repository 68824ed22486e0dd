"""Group norm of batches of short graphs with more groups than a block has room for (instance norms, pairs of channels): a tile
of channels holds no more of them than the arrays of a block."""
import pytest
import torch

from test_gpu_norm import BF16, DEV, F32, check, empty_graph, inputs, ragged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("F,groups", [(129, 129), (136, 136), (256, 256), (512, 256), (512, 512), (602, 602), (1024, 512),
                                      (1024, 1024), (516, 172)])
@pytest.mark.parametrize("graphs,rows", [(300, 11), (2048, 20), (1000, 64)])
def test_batches_with_many_groups(F, groups, graphs, rows, act):
    n = graphs * rows
    offsets = ragged(n, graphs, 17, F + graphs)
    g = empty_graph(n)
    g.dg_graph_set_batch(offsets)
    for x_type, y_type in ((F32, F32), (BF16, BF16), (BF16, F32)):
        X, dY, w, b = inputs(n, F, x_type, y_type, F)
        X[offsets[-1]:], dY[offsets[-1]:] = float("nan"), float("nan")   # padding is not read
        check(g, X, dY, groups, w, b, act, offsets)


def test_a_batch_of_equal_graphs_repeats():
    graphs, rows, F = 2048, 64, 256
    n = graphs * rows
    g = empty_graph(n)
    g.dg_graph_set_batch(torch.arange(0, n + 1, rows))
    X, dY, w, b = inputs(n, F, F32, F32, 1)
    first = check(g, X, dY, F, w, b, "relu", list(range(0, n + 1, rows)))
    again = check(g, X, dY, F, w, b, "relu", list(range(0, n + 1, rows)))
    for a, c in zip((first[0], first[1], *first[2]), (again[0], again[1], *again[2])):
        assert torch.equal(a, c)
