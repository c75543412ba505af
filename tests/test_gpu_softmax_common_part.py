"""g_in of gs_softmax_loss on tables whose rows share a large part.

g_in[i] = f sum_{j != t} p_j (c_j - c_t).  With probabilities of 16 bits, p_j (1 + e_j), |e_j| <= u, the sum and the context's
share have to be of the same rounded numbers: then it is off by u sum p_j |c_j - c_t|, not by u times the rows' common part.
What else is in the bound: r = 2 dz + 100 v from the scores as in test_gpu_softmax.py, fp32 sums of n terms on either side,
(n + 8) v (sum p_j |c_j| + (1 - p_t) |c_t|), and the result's own rounding.  binary16 also: probabilities below its normal
numbers, scaled by 2^11 at least under their row's largest, are off by half its least step, 2^-25, on both sides alike."""
import math

import pytest
import torch

from test_gpu_softmax import DEV, DTYPES, V, gs, make, reference  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(1, 3, 64), (50, 5, 64), (300, 40, 200), (64, 700, 128)])
@pytest.mark.parametrize("masked", [False, True])
def test_rows_with_a_large_common_part(gs, fmt, n, nodes, dim, masked):  # noqa: F811
    g = torch.Generator().manual_seed(n + nodes)
    middle = 24.0 * torch.sign(torch.randn(dim, generator=g))
    w_out = (middle + 0.5 * torch.randn(nodes, dim, generator=g)).to(DTYPES[fmt])
    w_in = (0.8 / math.sqrt(dim) * torch.randn(n, dim, generator=g)).to(DTYPES[fmt])
    c, t = torch.arange(n, dtype=torch.int32), torch.randint(0, nodes, (n,), generator=g, dtype=torch.int32)
    bias = None
    if masked:
        bias = torch.randn(nodes, generator=g)
        bias[1] = -math.inf
        t[t == 1] = 0
    *_, dz = reference(w_in, w_out, c, t, bias)
    h, w = w_in.double(), w_out.double()
    z = h @ w.T + (0.0 if bias is None else bias.double())
    at = t.long()[:, None]
    others = torch.softmax(z, 1).scatter(1, at, 0.0)
    from_t = w[None] - w[t.long()][:, None]                             # c_j - c_t
    f = 0.5
    want = f * torch.einsum("ij,ijd->id", others, from_t)
    size = f * torch.einsum("ij,ijd->id", others, from_t.abs())
    whole = f * (others @ w.abs() + others.sum(1, keepdim=True) * w[t.long()].abs())
    u = torch.finfo(DTYPES[fmt]).eps / 2
    least = 2.0 ** -25 if fmt == "f16" else 0.0
    low = f * least * 2.0 ** -11 * others.amax(1, keepdim=True) * from_t.abs().sum(1)
    bound = (2 * dz + 100 * V + (u if fmt != "f32" else 0.0)) * size + (nodes + 8) * V * whole + low
    bound = bound + u * (want.abs() + bound) + least
    _, got, _ = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)), bias=None if bias is None else bias.to(DEV), grad_scale=f)
    off = (got.cpu().double() - want).abs()
    assert torch.all(off <= bound), float((off / bound).max())
