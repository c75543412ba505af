"""gs_softmax_loss and gs_scores where a workgroup streams three tiles and more, so that every buffer is filled again: odd and
even numbers of tiles, offsets, and maxima that move all the way.  Bounds as in test_gpu_softmax.py; the definition's products
are taken on the GPU, in 64 bits."""
import math

import pytest
import torch

from test_gpu_softmax import DEV, DTYPES, V, gs, make, reference  # noqa: F401

pytestmark = pytest.mark.gpu


# pairs x nodes is some 15 million: 512 workgroups (fp32 from 200 columns on: 256) share it, 128 kept rows and three to twelve tiles each
@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(3000, 5000, 64), (5003, 3001, 128), (2601, 5200, 208), (1100, 14_001, 24)])
@pytest.mark.parametrize("offsets", ["none", "rising", "masked"])
def test_loss_and_gradients_over_many_tiles(gs, fmt, n, nodes, dim, offsets):  # noqa: F811
    w_in, w_out, c, t = make(n, nodes, dim, fmt, rows=700)
    t[::9] = -1
    bias = torch.zeros(nodes)
    if offsets == "rising":                    # the largest score moves with every tile
        bias = torch.linspace(-40.0, 0.0, nodes)
    elif offsets == "masked":
        bias = torch.randn(nodes, generator=torch.Generator().manual_seed(1))
        out = torch.rand(nodes, generator=torch.Generator().manual_seed(2)) < 0.3
        out[64:192], out[5] = True, False      # whole tiles among them
        bias[out] = -math.inf
        t = torch.where((t >= 0) & out[t.clamp(min=0).long()], 5, t)
    w_in, w_out, c, t, bias = (x.to(DEV) for x in (w_in, w_out, c, t, bias))
    f = 1.0 / n
    loss, g_in, g_out, g_in_abs, g_out_abs, dz = reference(w_in, w_out, c, t, bias, 0.75, f)
    call = lambda **k: gs.gs_softmax_loss(w_in, w_out, c, t, bias=bias if offsets != "none" else None, scale=0.75, grad_scale=f, **k)  # noqa: E731
    got, gi, go = call()
    live = t >= 0
    near = (2 * dz + 80 * V + 4 * V * loss.abs())[live]
    assert torch.all(got[~live] == 0) and torch.all((got.double() - loss).abs()[live] <= near)
    assert torch.all((call(want_grad=False)[0].double() - loss).abs()[live] <= near)
    u = torch.finfo(DTYPES[fmt]).eps / 2
    r = 2 * dz + 100 * V + (u if fmt != "f32" else 0.0)
    least = 2.0 ** -25 if fmt == "f16" else 0.0
    for have, want, size, terms in ((gi, g_in, g_in_abs, nodes), (go, g_out, g_out_abs, n)):
        bound = (r + terms * V + 4 * V) * size[0] + size[1]
        bound = bound + u * (want.abs() + bound) + least
        assert torch.all((have.double() - want).abs() <= bound), float(((have.double() - want).abs() - bound).max())
    again = call()
    assert torch.equal(again[0], got) and torch.equal(again[1], gi) and torch.equal(again[2], go)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(96, 70_000, 64), (100, 70_001, 200), (135, 131_075, 32), (133, 131_200, 128), (161, 66_000, 256)])
@pytest.mark.parametrize("offsets", [False, True])
def test_scores_over_many_tiles(gs, fmt, n, nodes, dim, offsets):  # noqa: F811
    """512 workgroups and more along the nodes, three to six tiles of 32 centres each; the last has 4, 5, 7, 1 or all."""
    w_in, w_out, c, _ = make(n, nodes, dim, fmt, rows=50)
    c[n // 2], c[n - 1] = 50, -1
    bad = torch.zeros(n, dtype=torch.bool)
    bad[n // 2] = bad[n - 1] = True
    bias, out = torch.zeros(nodes), torch.zeros(nodes, dtype=torch.bool)
    if offsets:
        bias = torch.randn(nodes, generator=torch.Generator().manual_seed(3))
        out = torch.rand(nodes, generator=torch.Generator().manual_seed(4)) < 0.2
        w_out[out] = math.nan
    w_in, w_out, c, bias, bad, out = (x.to(DEV) for x in (w_in, w_out, c, bias, bad, out))
    got = gs.gs_scores(w_in, w_out, c, bias=bias.masked_fill(out, -math.inf) if offsets else None, scale=1.5)
    assert torch.all(got[:, out] == -math.inf) and torch.isnan(got[bad][:, ~out]).all()
    h, w = w_in.double()[c.long()[~bad]], w_out.double()[~out]
    want = 1.5 * (h @ w.T) + bias.double()[~out]
    bound = (dim + 4) * V * 1.5 * (h.abs() @ w.abs().T) + 4 * V * want.abs() + 2 * V * bias.abs().max()
    assert torch.all((got[~bad][:, ~out].double() - want).abs() <= bound)
