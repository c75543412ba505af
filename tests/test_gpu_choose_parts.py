"""gs_sample_scores where a workgroup of a shared row takes more parts than it has waves, and where a part is longer than one
histogram along the index (rows beyond four million scores).  The definition in numpy's long doubles (64 bits of mantissa):
their sums of 8.5 million weights are off by 5e-13 of the sum at most, those of the call by 2^-62 a weight and 1e-15 of the sum:
one random number in a hundred thousand would lie that near to a border.  Ids have to be equal, probabilities within half a step
of fp32."""
import math

import numpy as np
import pytest
import torch

from test_gpu_choose import DEV, gs, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu


def choose(z, u, temperature, k, top_p, min_p):
    rank = np.flatnonzero(z > -np.inf)
    rank = rank[np.argsort(-z[rank], kind="stable")]
    w = np.exp((z[rank].astype(np.longdouble) - z[rank[0]]) / np.longdouble(temperature))
    if k > 0:
        rank, w = rank[:k], w[:k]
    if top_p < 1:
        m = max(1, int((np.cumsum(w) - w < np.longdouble(top_p) * w.sum()).sum()))
        rank, w = rank[:m], w[:m]
    if min_p > 0:
        m = int((w >= min_p).sum())
        rank, w = rank[:m], w[:m]
    back = np.argsort(rank)
    rank, w = rank[back], w[back]
    j = min(int(np.searchsorted(np.cumsum(w), np.longdouble(u) * w.sum(), side="right")), w.size - 1)
    return int(rank[j]), float(w[j] / w.sum())


def check(gs, z, u, temperature, k, top_p, min_p):  # noqa: F811
    par = dict(temperature=torch.tensor(temperature, dtype=torch.float32), top_k=torch.tensor(k, dtype=torch.int32),
               top_p=torch.tensor(top_p, dtype=torch.float32), min_p=torch.tensor(min_p, dtype=torch.float32))
    ids, probs = gs.gs_sample_scores(z.to(DEV), u.to(DEV), **{a: b.to(DEV) for a, b in par.items()})
    zz = z.double().numpy()
    for r in range(z.shape[0]):
        want, p = choose(zz[r], float(u[r]), *(float(par[a][r]) if a != "top_k" else int(par[a][r]) for a in ("temperature", "top_k", "top_p", "min_p")))
        assert int(ids[r]) == want, (r, int(ids[r]), want)
        assert abs(float(probs[r]) - p) <= 2.0 ** -24 * p + 1e-12, r


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_many_parts_for_each_workgroup(gs, fmt):  # noqa: F811
    rows, n = 256, 100_003
    z, u = rows_of(rows, n, fmt, seed=5)
    check(gs, z, u, [1.0, 0.7, 1.3, 2.0] * 64, [0, 0, 50, 0, 0, 900, 0, 0] * 32, [1.0, 0.9, 0.8, 0.99, 0.5, 1.0, 1.0, 0.95] * 32, [0.0, 0.0, 0.01, 0.002] * 64)


@pytest.mark.parametrize("fmt,n", [("f32", 4_300_007), ("bf16", 8_500_001), ("f16", 4_300_007)])
def test_rows_of_millions(gs, fmt, n):  # noqa: F811
    z, _ = rows_of(1, n, fmt, seed=6)
    z = z.expand(4, n).contiguous()
    z[3, : n - 3] = -math.inf
    check(gs, z, torch.tensor([0.999, 0.3, 0.5, 0.6]), [2.0, 0.8, 1.0, 1.0], [0, 0, 700, 0], [1.0, 0.9, 0.8, 0.9], [0.0, 0.001, 0.0, 0.0])
