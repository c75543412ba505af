"""gs_softmax_loss: pairs without gradient beside node rows that hold infinities and NaN."""
import math

import pytest
import torch

from test_gpu_softmax import DEV, gs, make  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(1, 40, 64), (70, 300, 72), (3000, 70, 200), (300, 40_000, 256)])
@pytest.mark.parametrize("offsets", [False, True])
def test_pairs_without_gradient_beside_rows_of_no_numbers(gs, fmt, n, nodes, dim, offsets):  # noqa: F811
    """No pair of the batch has a gradient: every row of both is zero, whatever a node's row holds."""
    w_in, w_out, c, t = make(n, nodes, dim, fmt)
    w_out[0], w_out[nodes // 2, dim - 1], w_out[nodes - 1, 0] = math.nan, math.inf, -math.inf
    t[:] = -1
    if n > 3:
        c[1], t[1], c[2], t[2], t[3] = nodes, 5, -1, 0, nodes
    bias = torch.linspace(-1, 1, nodes).to(DEV) if offsets else None
    loss, gi, go = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)), bias=bias)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[1:4] = n > 3
    assert torch.equal(loss.cpu().isnan(), bad) and torch.all(loss.cpu()[~bad] == 0)
    assert torch.all(gi == 0) and torch.all(go == 0)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes", [(5, 90), (700, 300)])
def test_a_node_at_minus_infinity(gs, fmt, n, nodes):  # noqa: F811
    """A score of -infinity by the node's row: no weight and no gradient of its own, and the other rows' as if it were masked."""
    w_in, w_out, c, t = make(n, nodes, 64, fmt)
    w_in = w_in.abs() + 0.25
    t = torch.where(t == 7, t + 1, t)
    if n > 5:
        t[3::11] = -1
    clean = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)), bias=torch.zeros(nodes).index_fill_(0, torch.tensor([7]), -math.inf).to(DEV))
    w_out[7, 10] = -math.inf
    loss, _, go = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)))
    assert torch.allclose(loss, clean[0], rtol=1e-5, atol=1e-5) and torch.all(go[7] == 0)
    assert torch.isfinite(go).all() and torch.allclose(go.float(), clean[2].float(), rtol=2.0 ** -6, atol=1e-4)
