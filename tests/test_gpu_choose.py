"""gs_sample_scores against the definition in 64 bits (numpy: sorted, cut, searched): the ids have to be equal, the
probabilities within half a step of fp32 of the fp64 value (2^-24 relative, and 1e-12 for the sums' own order)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def gs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2407_15452_amd import binding
    binding.lib()
    return binding


def choose(z, u, temperature=1.0, k=0, top_p=1.0, min_p=0.0):
    """(id, probability) of one row; z float64."""
    may = np.flatnonzero(z > -np.inf)
    if not may.size:
        return -1, 0.0
    rank = may[np.argsort(-z[may], kind="stable")]
    if temperature == 0:
        return int(rank[0]), 1.0
    top = z[rank[0]]
    with np.errstate(all="ignore"):
        w = np.where(z[rank] == top, 1.0, np.exp((z[rank] - top) / np.float64(temperature)))
    if k > 0:
        rank, w = rank[:k], w[:k]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        m = max(1, int((before < float(top_p) * w.sum()).sum()))
        rank, w = rank[:m], w[:m]
    if min_p > 0:
        m = int((w >= min(float(min_p), 1.0)).sum())
        rank, w = rank[:m], w[:m]
    back = np.argsort(rank)
    rank, w = rank[back], w[back]
    sums = np.cumsum(w)
    over = np.flatnonzero((sums > float(u) * w.sum()) & (w > 0))
    j = over[0] if over.size else np.flatnonzero(w > 0)[-1]
    return int(rank[j]), w[j] / w.sum()


def check(gs, z, u, temperature=None, top_k=None, top_p=None, min_p=None):
    rows = z.shape[0]
    dev = lambda x, t=torch.float32: None if x is None else torch.as_tensor(x, dtype=t).to(DEV)  # noqa: E731
    par = {"temperature": dev(temperature), "top_k": dev(top_k, torch.int32), "top_p": dev(top_p), "min_p": dev(min_p)}
    ids, probs = gs.gs_sample_scores(z.to(DEV), dev(u), **par)
    again = gs.gs_sample_scores(z.to(DEV), dev(u), **par)
    assert torch.equal(ids, again[0]) and torch.equal(probs, again[1])
    host = {k: (v.cpu().numpy() if v is not None else None) for k, v in par.items()}
    zz, uu = z.double().numpy(), torch.as_tensor(u, dtype=torch.float32).numpy()
    for r in range(rows):
        arg = {}
        for name, to in (("temperature", "temperature"), ("top_k", "k"), ("top_p", "top_p"), ("min_p", "min_p")):
            if host[name] is not None:
                arg[to] = host[name][r]
        want_id, want_p = choose(zz[r], uu[r], **arg)
        assert int(ids[r]) == want_id, (r, arg, float(uu[r]), int(ids[r]), want_id)
        assert abs(float(probs[r]) - want_p) <= 2.0 ** -24 * want_p + 1e-12, r
    return ids, probs


def rows_of(rows, n, fmt, seed=0, spread=2.0, masked=0.1):
    g = torch.Generator().manual_seed(seed * 31 + rows * 1009 + n)
    z = spread * torch.randn(rows, n, generator=g)
    z[torch.rand(rows, n, generator=g) < masked] = -math.inf
    return z.to(DTYPES[fmt]), torch.rand(rows, generator=g)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (5, 2), (40, 63), (33, 64), (20, 65), (16, 1000), (9, 1025), (5, 5003), (3, 24_576),
                                    (3, 24_577), (2, 70_001)])
@pytest.mark.parametrize("filters", ["", "k", "p", "m", "kp", "kpm"])
def test_filters(gs, fmt, rows, n, filters):
    z, u = rows_of(rows, n, fmt)
    g = torch.Generator().manual_seed(n)
    k = (torch.rand(rows, generator=g) * min(n, 300)).int() if "k" in filters else None       # 0 among them: no limit
    check(gs, z, u, temperature=0.5 + torch.rand(rows, generator=g), top_k=k,
          top_p=0.3 + 0.69 * torch.rand(rows, generator=g) if "p" in filters else None,
          min_p=0.2 * torch.rand(rows, generator=g) if "m" in filters else None)


@pytest.mark.parametrize("n", [7, 300, 3000, 30_000])
def test_ties_go_to_the_lowest_index(gs, n):
    """Scores of few values: cuts fall among equal ones."""
    g = torch.Generator().manual_seed(n)
    rows = 24
    z = torch.randint(-2, 3, (rows, n), generator=g).float() * 0.5
    u = torch.rand(rows, generator=g)
    check(gs, z, u, top_k=1 + (torch.rand(rows, generator=g) * n).int())
    check(gs, z, u, top_p=torch.rand(rows, generator=g))
    check(gs, z, u, top_k=1 + (torch.rand(rows, generator=g) * n).int(), top_p=torch.rand(rows, generator=g), min_p=0.4 * torch.rand(rows, generator=g))
    check(gs, torch.zeros(rows, n), u, top_k=1 + (torch.rand(rows, generator=g) * n).int())
    check(gs, z, u, temperature=torch.zeros(rows))
    ids, _ = gs.gs_sample_scores(torch.tensor([[0.0, -0.0, 0.0]], device=DEV).repeat(3, 1), torch.tensor([0.0, 0.4, 0.9], device=DEV))
    assert ids.tolist() == [0, 1, 2]


def test_borders_of_the_random_number(gs):
    """Weights of 1: sums are whole numbers and u * sum is exact, so a border belongs to the node after it."""
    z = torch.zeros(6, 4)
    z[:, 2] = -math.inf
    u = torch.tensor([0.0, math.nan, 1.0, -0.5, 2.0, 0.99999994])
    ids, probs = gs.gs_sample_scores(z.to(DEV), u.to(DEV))
    assert ids.tolist() == [0, 3, 3, 0, 3, 3] and torch.allclose(probs.cpu(), torch.full((6,), 1 / 3))
    z = torch.zeros(5, 4).to(DEV)
    ids, _ = gs.gs_sample_scores(z, torch.tensor([0.0, 0.25, 0.5, 0.75, 0.24999999], device=DEV))
    assert ids.tolist() == [0, 1, 2, 3, 0]


def test_rows_without_answers_and_values_that_are_no_numbers(gs):
    inf, nan = math.inf, math.nan
    z = torch.tensor([[-inf, -inf, -inf], [nan, nan, -inf], [nan, 1.0, nan], [inf, 3.0, inf], [-inf, -3e38, -inf], [3e38, -3e38, 0.0]])
    u = torch.tensor([0.5, 0.5, 0.9, 0.6, 0.3, 0.999])
    for kw in ({}, {"top_k": [2] * 6}, {"top_p": [0.9] * 6}, {"min_p": [0.5] * 6}, {"top_k": [2] * 6, "top_p": [0.9] * 6}):
        par = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device=DEV) for k, v in kw.items()}
        ids, probs = gs.gs_sample_scores(z.to(DEV), u.to(DEV), **par)
        assert ids.tolist() == [-1, -1, 1, 2 if kw.get("top_p", [1])[0] != 0.5 else 0, 1, 0]
        assert probs.tolist() == [0.0, 0.0, 1.0, 0.5, 1.0, 1.0]


def test_limits_that_do_not_limit(gs):
    z, u = rows_of(8, 500, "f32")
    plain = gs.gs_sample_scores(z.to(DEV), u.to(DEV))
    off = {"top_k": torch.tensor([0, -5, 500, 501, 2 ** 31 - 1, 0, 0, 0], dtype=torch.int32, device=DEV),
           "top_p": torch.tensor([1.0, 2.0, math.nan, math.inf] * 2, device=DEV),
           "min_p": torch.tensor([0.0, -1.0, math.nan, -math.inf] * 2, device=DEV), "temperature": torch.ones(8, device=DEV)}
    got = gs.gs_sample_scores(z.to(DEV), u.to(DEV), **off)
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    one = {"top_p": torch.tensor([0.0, -1.0, 1e-30, 1e-9] * 2, device=DEV)}
    best = gs.gs_sample_scores(z.to(DEV), u.to(DEV), temperature=torch.zeros(8, device=DEV))
    assert torch.equal(gs.gs_sample_scores(z.to(DEV), u.to(DEV), **one)[0], best[0])
    assert torch.equal(gs.gs_sample_scores(z.to(DEV), u.to(DEV), min_p=torch.full((8,), 7.0, device=DEV))[0], best[0])


def test_temperatures(gs):
    z, u = rows_of(7, 900, "f32")
    check(gs, z, u, temperature=[0.0, 1e-30, 1e-3, 0.1, 10.0, 1e30, math.inf], top_k=[50] * 7)
    check(gs, z, u, temperature=[0.0, 1e-30, 1e-3, 0.1, 10.0, 1e30, math.inf], top_p=[0.9] * 7)
    ids, probs = gs.gs_sample_scores(z.to(DEV), u.to(DEV), temperature=torch.tensor([-1.0, math.nan] + [1.0] * 5, device=DEV))
    assert ids.tolist()[:2] == [-1, -1] and torch.isnan(probs[:2]).all() and torch.all(ids[2:] >= 0)


@pytest.mark.parametrize("filters", ["k", "p", "kp"])
def test_scores_far_from_evenly_spread(gs, filters):
    """One score of 1e30, scores around zero of either sign down to the least magnitudes, and a dense cluster."""
    g = torch.Generator().manual_seed(9)
    n, rows = 6000, 12
    z = torch.randn(rows, n, generator=g)
    z[0:3, 17] = 1e30
    z[3:6] = z[3:6] * torch.pow(10.0, -40 * torch.rand(3, n, generator=g))
    z[6:9] = 5.0 + z[6:9] * 1e-5
    z[9:12, 100:] = -1e30
    u = torch.rand(rows, generator=g)
    check(gs, z, u, top_k=[500] * rows if "k" in filters else None, top_p=[0.8] * rows if "p" in filters else None)


def test_chosen_as_often_as_likely(gs):
    """Evenly spaced random numbers: each node is chosen p_j * rows times, up to one at each border."""
    rows, n = 4096, 37
    z = torch.randn(1, n, generator=torch.Generator().manual_seed(4))
    u = (torch.arange(rows) + 0.5) / rows
    ids, _ = gs.gs_sample_scores(z.repeat(rows, 1).to(DEV), u.to(DEV))
    hits = torch.bincount(ids.cpu().long(), minlength=n).double()
    assert torch.all((hits - rows * torch.softmax(z[0].double(), 0)).abs() <= 1.0)


def test_graph_replays_on_another_stream(gs):
    z, u = (x.to(DEV) for x in rows_of(16, 3000, "f32"))
    par = {"top_k": torch.full((16,), 40, dtype=torch.int32, device=DEV), "top_p": torch.full((16,), 0.9, device=DEV)}
    ws = torch.empty(gs.gs_sample_scores_workspace_bytes(16, 3000), dtype=torch.uint8, device=DEV)
    ids, probs = torch.empty(16, dtype=torch.int32, device=DEV), torch.empty(16, device=DEV)
    call = lambda: gs.gs_sample_scores(z, u, ids_out=ids, probs_out=probs, ws=ws, **par)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        u.copy_(torch.rand(16, generator=torch.Generator().manual_seed(k)))
        want = gs.gs_sample_scores(z, u, **par)
        ids.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, want[0]) and torch.equal(probs, want[1])


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 24_577), (2, 262_147), (7, 100_003), (3, 131_072)])
def test_long_rows_shared_by_several_workgroups(gs, fmt, rows, n):
    """Rows of mixed limits in one call: none, top-k, top-p, both, greedy, k beyond the row, everything left out."""
    g = torch.Generator().manual_seed(rows + n)
    z, _ = rows_of(rows * 8, n, fmt, seed=2)
    if rows > 2:
        z[5] = -math.inf
        z[6, : n - 1] = -math.inf
    u = torch.rand(rows * 8, generator=g)
    u[0], u[1] = 0.0, 1.0
    k = torch.tensor([0, 50, 0, 700, 1, n + 5, n - 1, 3000] * rows, dtype=torch.int32)
    p = torch.tensor([1.0, 1.0, 0.9, 0.5, 0.3, 0.8, 0.999, 0.05] * rows)
    t = torch.tensor([1.0, 0.7, 1.3, 1.0, 0.0, 1.0, 2.0, 0.5] * rows)
    check(gs, z, u, temperature=t, top_k=k, top_p=p, min_p=[0.0, 0.01, 0.0, 0.05] * (2 * rows))
    check(gs, z, u, temperature=t, top_k=k)
    check(gs, z, u, temperature=t, top_p=p)
    check(gs, z, u, min_p=[0.0, 0.01, 0.2, 1.0] * (2 * rows))


@pytest.mark.parametrize("top_k,top_p", [(None, 0.6), (40_000, None), (40_000, 0.6), (7, None), (1_000_000, 0.5)])
def test_long_rows_of_equal_scores(gs, top_k, top_p):
    """More elements fall on the cut than a row's list has room for."""
    rows, n = 4, 60_000
    z = torch.zeros(rows, n)
    z[1] = torch.randint(0, 3, (n,), generator=torch.Generator().manual_seed(1)).float()
    z[2, ::2] = 1e-3 * torch.arange(n // 2) / n
    z[3, 0] = 1e30
    u = torch.tensor([0.3, 0.6, 0.9, 0.99])
    check(gs, z, u, top_k=None if top_k is None else [top_k] * rows, top_p=None if top_p is None else [top_p] * rows)


@pytest.mark.parametrize("n", [9000, 120_000])
@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_lists_of_more_than_one_histogram(gs, n, fmt):
    """Thousands of nodes kept by top-k, or equal to the score that top-p cuts at."""
    z, u = rows_of(6, n, fmt, seed=11)
    check(gs, z, u, top_k=[2047, 2048, 2049, 4095, 4096, 4097])
    check(gs, z, u, top_k=[2047, 2048, 2049, 3900, 4096, 4097], top_p=[0.999, 0.99, 0.9, 0.9999, 0.5, 0.7], min_p=[0.0, 1e-4] * 3)
    z = torch.round(z * 4) / 4                       # some hundred values
    check(gs, z, u, top_p=[0.5, 0.7, 0.9, 0.95, 0.99, 0.999])
    check(gs, z, u, top_k=[1500, 2500, 3500, 4000, 5000, 8000], top_p=[0.5, 0.7, 0.9, 0.95, 0.99, 0.999])


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [8193, 12_001, 16_383])
def test_long_rows_of_one_workgroup(gs, fmt, n):
    """Bins of several neighbouring indices: the weights of a piece are added up before they go to a bin."""
    z, u = rows_of(7, n, fmt, seed=11, masked=0.3)
    u[0], u[1] = 0.0, float(np.nextafter(np.float32(1.0), np.float32(0.0)))
    z[2, :-1] = -math.inf                                  # the last alone
    check(gs, z, u)
    check(gs, z, u, temperature=[0.5, 1.0, 2.0, 0.25, 1.5, 4.0, 0.7], min_p=[0.0, 0.01, 0.5, 1.0, 0.2, 0.001, 0.05])
