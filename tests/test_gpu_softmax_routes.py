"""gs_softmax_loss with one gradient alone, on batches in few and in many parts: the routes that a null g_in or g_out takes.  Bounds
as in test_gpu_softmax.py; with g_in alone the same bits come out as with both."""
import math

import pytest
import torch

from test_gpu_softmax import DEV, DTYPES, V, check, gs, make, reference  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(3, 5000, 64), (300, 2000, 200), (9000, 70, 72), (70_000, 300, 32), (5, 7, 128)])
@pytest.mark.parametrize("offsets", [False, True])
def test_one_gradient_alone(gs, fmt, n, nodes, dim, offsets):  # noqa: F811
    w_in, w_out, c, t = make(n, nodes, dim, fmt, rows=90)
    t[1::7] = -1
    bias = None
    if offsets:
        bias = torch.randn(nodes, generator=torch.Generator().manual_seed(1))
        bias[::5] = -math.inf
        t = torch.where((t >= 0) & (t % 5 == 0), t + 1, t)
    loss, gi, go = check(gs, w_in, w_out, c, t, fmt, bias=bias, grad_scale=1.0 / n)
    d = [x.to(DEV) for x in (w_in, w_out, c, t)]
    db = None if bias is None else bias.to(DEV)
    ws = torch.full((gs.gs_softmax_loss_workspace_bytes(n, nodes, dim, gs._table_dtype(w_in)),), 255, dtype=torch.uint8, device=DEV)
    l1, g1, none = gs.gs_softmax_loss(*d, bias=db, grad_scale=1.0 / n, want_grad="in", ws=ws)
    assert none is None and torch.equal(l1.cpu(), loss) and torch.equal(g1.cpu(), gi)
    ws.fill_(255)
    l2, none, g2 = gs.gs_softmax_loss(*d, bias=db, grad_scale=1.0 / n, want_grad="out", ws=ws)
    assert none is None and torch.equal(l2, gs.gs_softmax_loss(*d, bias=db, want_grad=False)[0])
    want_loss, _, want, _, size, dz = reference(w_in, w_out, c, t, bias, 1.0, 1.0 / n)
    live = t >= 0
    assert torch.all((l2.cpu().double() - want_loss).abs()[live] <= 2 * dz + 80 * V + 4 * V * want_loss.abs()[live])
    u = torch.finfo(DTYPES[fmt]).eps / 2
    bound = (2 * dz + 100 * V + (u if fmt != "f32" else 0.0) + (n + 4) * V) * size[0] + size[1]
    bound = bound + u * (want.abs() + bound) + (2.0 ** -25 if fmt == "f16" else 0.0)
    assert torch.all((g2.cpu().double() - want).abs() <= bound)
    into = torch.full_like(g2, 3.0)
    assert gs.gs_softmax_loss(*d, bias=db, grad_scale=1.0 / n, want_grad="out", g_out=into)[2] is into and torch.equal(into, g2)
