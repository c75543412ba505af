"""How far 16-bit scores of wide rows are off as a whole.

Per score the bound of test_gpu_scores_q8.py is that of the worst case, 7 * 2^-13 of the products' sizes, under which a few wrong products of
thousands would pass.  Here the root of the mean square over all scores is bounded, for Gaussian rows: what the 8-bit instruction
drops by 2^-16 of the products' sizes (gs.h), the rounding to 16 bits by half a step of each score, and the fp32 sums by 2^-23 of a partial
sum for each of dim + 2 operations, where a sum of some of the columns, which are independent, has a smaller mean square than the
whole.  Means add up at most.  With 8192 columns and scores of size 1 that is 9e-4 + 5e-4 (fp16) + 1e-3, and one product is 1.1e-2, so that one left out or
taken twice in every score shows, as the last test does with the oracle."""
import pytest
import torch

from test_gpu_scores_q8 import DEV, HALF_STEP, TORCH, gs, table, values  # noqa: F401

pytestmark = pytest.mark.gpu


def rms(x):
    return float(x.double().square().mean().sqrt())


def products(t_in, t_out, ids):
    h, c = values(t_in)[ids.long()], values(t_out)
    return h @ c.T.contiguous(), h.abs() @ c.abs().T.contiguous(), h, c


def bound(want, size, dim, dtype):
    drop = 0.0 if dtype == "f32" else 2.0 ** -16
    return drop * rms(size) + (dim + 2) * 2.0 ** -23 * rms(want) + HALF_STEP[dtype] * rms(want)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("centers,nodes,dim", [(8, 4000, 1024), (32, 1000, 8192), (33, 4001, 256), (200, 3000, 200), (100, 2000, 1024), (300, 1500, 2048), (256, 600, 8192)])
def test_scores_as_a_whole(gs, centers, nodes, dim, dtype):  # noqa: F811
    t_in, t_out = table(gs, 300, dim, 21, spread=0.0), table(gs, nodes, dim, 22, spread=0.0)
    ids = torch.randperm(300, generator=torch.Generator().manual_seed(3))[:centers].to(torch.int32).to(DEV)
    want, size, h, c = products(t_in, t_out, ids)
    off = rms(gs.gs_scores_q8(t_in, t_out, ids, dtype=TORCH[dtype]).double() - want)
    assert off <= bound(want, size, dim, dtype), (off, bound(want, size, dim, dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_one_product_more_or_less_shows(gs, dtype):  # noqa: F811
    """Of the oracle, with the widest rows: a product left out, and one taken twice."""
    dim = 8192
    t_in, t_out = table(gs, 300, dim, 21, spread=0.0), table(gs, 600, dim, 22, spread=0.0)
    ids = torch.arange(256, dtype=torch.int32, device=DEV)
    want, size, h, c = products(t_in, t_out, ids)
    got = gs.gs_scores_q8(t_in, t_out, ids, dtype=TORCH[dtype]).double()
    for column in (0, 4097, dim - 1):
        for sign in (-1.0, 1.0):
            wrong = want + sign * h[:, column, None] * c[None, :, column]
            assert rms(got - wrong) > bound(wrong, size, dim, dtype)
