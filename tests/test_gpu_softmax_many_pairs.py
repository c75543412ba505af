"""gs_softmax_loss on more pairs than 24 bits count.  Bounds as in test_gpu_softmax.py."""
import pytest
import torch

from test_gpu_softmax import DEV, DTYPES, V, gs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_more_pairs_than_24_bits(gs, fmt):  # noqa: F811
    """A part of the table gradient sums 513 tiles of 64 pairs, and 512 parts are joined: fp32 sums of 33,400 terms."""
    n, nodes, dim = (1 << 24) + 300, 40, 8
    g = torch.Generator(device=DEV).manual_seed(3)
    w_in, w_out = (torch.randn(r, dim, generator=g, device=DEV).to(DTYPES[fmt]) for r in (1000, nodes))
    c = torch.randint(0, 1000, (n,), generator=g, device=DEV, dtype=torch.int32)
    t = torch.randint(-1, nodes, (n,), generator=g, device=DEV, dtype=torch.int32)
    loss, gi, go = gs.gs_softmax_loss(w_in, w_out, c, t)
    w = w_out.double()
    dz = (dim + 8) * V * float((w_in.double().abs() @ w.abs().T).amax())
    u = torch.finfo(DTYPES[fmt]).eps / 2
    r = 2 * dz + 100 * V + (u if fmt != "f32" else 0.0)
    want_out, size_out = (torch.zeros(nodes, dim, dtype=torch.float64, device=DEV) for _ in range(2))
    for lo in range(0, n, 1 << 21):
        h, x = w_in.double()[c[lo:lo + (1 << 21)].long()], t[lo:lo + (1 << 21)].long()
        z = h @ w.T
        live, at = x >= 0, x.clamp(min=0)[:, None]
        lse = torch.logsumexp(z, 1, keepdim=True)
        want = (lse - z.gather(1, at))[:, 0] * live
        assert torch.all((loss[lo:lo + (1 << 21)].double() - want).abs() <= 2 * dz + 80 * V + 4 * V * want)
        hot = torch.zeros_like(z).scatter_(1, at, 1.0)
        p = torch.exp(z - lse)
        coef, size = (p - hot) * live[:, None], (p + hot) * live[:, None]
        g_in, bound = coef @ w, (r + (nodes + 4) * V) * (size @ w.abs())
        assert torch.all((gi[lo:lo + (1 << 21)].double() - g_in).abs() <= bound + u * (g_in.abs() + bound) + 2.0 ** -126)
        want_out += coef.T @ h
        size_out += size.T @ h.abs()
    bound = (r + 33_400 * V) * size_out
    assert torch.all((go.double() - want_out).abs() <= bound + u * (want_out.abs() + bound))
