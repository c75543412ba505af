"""Tables, gradients and scores of more than 2^31 elements: gs_softmax_loss, gs_scores, gs_sample_scores.  Bounds as in
test_gpu_softmax.py; the definition's products are taken on the GPU, in 64 bits and pieces."""
import pytest
import torch

from test_gpu_softmax import DEV, V, gs  # noqa: F401

pytestmark = pytest.mark.gpu


def test_tables_scores_and_rows_beyond_31_bits(gs):  # noqa: F811
    """Element 2^31 lies in row 2^23 of the table and of its gradient, and in row 255 of the scores.  fp32 sums: 262 tiles of 32
    nodes a part at most, or 131 of 64, and 1024 parts at most: 9500 terms."""
    nodes, dim, n = (1 << 23) + 1029, 256, 3
    g = torch.Generator(device=DEV).manual_seed(4)
    w_in = (0.35 * torch.randn(300, dim, generator=g, device=DEV)).to(torch.bfloat16)
    w_out = torch.empty(nodes, dim, dtype=torch.bfloat16, device=DEV)
    step = 1 << 19
    for lo in range(0, nodes, step):
        part = w_out[lo:lo + step]
        part.copy_(0.35 * torch.randn(part.shape, generator=g, device=DEV))
    c = torch.tensor([7, 0, 299], dtype=torch.int32, device=DEV)
    t = torch.tensor([nodes - 1, (1 << 23) + 3, 5], dtype=torch.int32, device=DEV)
    loss, gi, go = gs.gs_softmax_loss(w_in, w_out, c, t)
    h = w_in.double()[c.long()]
    z = torch.cat([h @ w_out[lo:lo + step].double().T for lo in range(0, nodes, step)], 1)
    dz = (dim + 8) * V * float(max((h.abs() @ w_out[lo:lo + step].double().abs().T).amax() for lo in range(0, nodes, step)))
    lse = torch.logsumexp(z, 1, keepdim=True)
    want = (lse - z.gather(1, t.long()[:, None]))[:, 0]
    assert torch.all((loss.double() - want).abs() <= 2 * dz + 80 * V + 4 * V * want)
    p = torch.exp(z - lse)
    hot = torch.zeros_like(p).scatter_(1, t.long()[:, None], 1.0)
    u = 2.0 ** -8
    r = 2 * dz + 100 * V + u
    g_in, size_in = (torch.zeros(n, dim, dtype=torch.float64, device=DEV) for _ in range(2))
    for lo in range(0, nodes, step):
        w = w_out[lo:lo + step].double()
        coef, size = (p - hot)[:, lo:lo + step].contiguous(), (p + hot)[:, lo:lo + step].contiguous()
        g_in += coef @ w
        size_in += size @ w.abs()
        g_out, bound = coef.T @ h, (r + 8 * V) * (size.T @ h.abs()) + 2.0 ** -126 * (1 + h.abs().sum(0))
        assert torch.all((go[lo:lo + step].double() - g_out).abs() <= bound + u * (g_out.abs() + bound)), lo
    bound = (r + 9500 * V) * size_in + 2.0 ** -126 * nodes
    assert torch.all((gi.double() - g_in).abs() <= bound + u * (g_in.abs() + bound))
    del go, p, hot, z
    scores = gs.gs_scores(w_in, w_out, torch.arange(300, dtype=torch.int32, device=DEV))
    for row in (0, 128, 255, 256, 299):
        x = w_in[row:row + 1].double()
        for lo in range(0, nodes, step):
            w = w_out[lo:lo + step].double()
            want = x @ w.T
            assert torch.all((scores[row:row + 1, lo:lo + step].double() - want).abs() <= (dim + 4) * V * (x.abs() @ w.abs().T) + 4 * V * want.abs())
    u = torch.rand(300, generator=g, device=DEV)
    par = dict(temperature=(torch.arange(300, device=DEV) % 3).float(), top_k=(torch.arange(300, device=DEV) % 2 * 40).int(),
               top_p=torch.full((300,), 0.9, device=DEV))
    ids, probs = gs.gs_sample_scores(scores, u, **par)
    for row in (0, 1, 128, 254, 255, 256, 257, 297, 298, 299):
        one = gs.gs_sample_scores(scores[row:row + 1], u[row:row + 1], **{k: v[row:row + 1] for k, v in par.items()})
        assert int(one[0]) == int(ids[row]) and float(one[1]) == float(probs[row])
    greedy = torch.arange(0, 300, 3, device=DEV)
    assert torch.equal(scores[greedy].gather(1, ids[greedy].long()[:, None])[:, 0], scores[greedy].amax(1))
