"""gs_beam_select and gs_beam_reorder against their definitions, in 64 bits.

Parents and nodes are equal.  logp is fp64 rounded to fp32 once: half a step, 2^-24 of it, and what the definition leaves to p,
6e-14 (1 + |p| + |logp| + log n): weights 2^r, |r| <= 1/128, end with the fourth term of their series, and the fifth is
(log 2 / 128)^5 / 120 = 3.9e-14 of a weight, so of the sum at most, and of its logarithm; the exponents' roundings take 2^-52 |x| exp(x),
x <= 0, of the largest weight, less than 2^-53, and the handful of operations on p half a step of their numbers each, 2^-53."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")


@pytest.fixture(scope="module")
def gs():
    from paper_2407_15452_amd import binding
    binding.lib()
    return binding


def definition(scores, logp, beams, width, ended=None):
    """All candidates of a group in order: larger p, lower walk, larger score, lower node."""
    z = scores.double().cpu().numpy()
    before = logp.double().cpu().numpy()
    groups, n = len(before) // beams, z.shape[1]
    parents, nodes, out = np.full((groups, width), -1), np.full((groups, width), -1), np.full((groups, width), -np.inf)
    for g in range(groups):
        found = []
        for b in range(beams):
            r = g * beams + b
            if not before[r] > -np.inf:
                continue
            if ended is not None and bool(ended[r]):
                found.append((-before[r], b, 0.0, -1))
                continue
            at = np.flatnonzero(z[r] > -np.inf)
            if not at.size:
                continue
            s = z[r][at]
            top = s.max()
            below = np.where(s == top, 0.0, s - top) if np.isfinite(top) else np.where(s == top, 0.0, -np.inf)
            p = before[r] + (below - math.log(math.fsum(np.exp(below))))
            order = np.lexsort((at, -s))[:width]
            found += [(-p[o], b, -s[o], at[o]) for o in order if p[o] > -np.inf]
        for t, (p, b, _, a) in enumerate(sorted(found)[:width]):
            parents[g, t], nodes[g, t], out[g, t] = b, a, -p
    return parents, nodes, out


def check(gs, scores, logp, beams, width, ended=None):
    got = gs.gs_beam_select(scores, logp, beams, width, ended=ended)
    want = definition(scores, logp, beams, width, ended)
    assert [x.dtype for x in got] == [torch.int32, torch.int32, torch.float32]
    parents, nodes, p = (x.cpu().numpy() for x in got)
    assert np.array_equal(parents, want[0])
    assert np.array_equal(nodes, want[1])
    fine = np.isfinite(want[2])
    assert np.array_equal(p[~fine], want[2][~fine].astype(np.float32))
    size, before = np.abs(want[2][fine]), float(logp[torch.isfinite(logp)].abs().max()) if bool(torch.isfinite(logp).any()) else 0.0
    assert (np.abs(p[fine].astype(np.float64) - want[2][fine]) <= 2.0 ** -24 * size + 6e-14 * (1 + size + before + math.log(scores.shape[1])) + 2.0 ** -150).all()
    return got


def some(rows, n, dtype, seed, masked=0.1, spread=2.0):
    gen = torch.Generator().manual_seed(seed)
    z = spread * torch.randn(rows, n, generator=gen)
    z[torch.rand(rows, n, generator=gen) < masked] = -INF
    return z.to(TORCH[dtype]).to(DEV), (-20 * torch.rand(rows, generator=gen)).to(DEV)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("groups,beams,n,width", [
    (1, 1, 1, 1), (1, 1, 7, 3), (2, 3, 1, 4), (3, 2, 5, 16), (1, 4, 255, 4), (5, 3, 1023, 1), (4, 8, 1025, 8), (300, 1, 100, 5), (1, 1, 70_001, 16),
    (7, 4, 4099, 32), (2, 16, 3001, 64), (1, 32, 20_000, 100), (1, 2, 300_007, 10), (1, 256, 300, 256), (2, 1, 5000, 256), (1, 5, 16_384, 256),
    (1, 5, 16_385, 200), (1, 1, 1_000_003, 64), (600, 2, 9, 2), (40, 8, 40_000, 4), (3, 7, 32_769, 128), (1, 200, 17, 3), (64, 16, 8193, 12)])
def test_select(gs, groups, beams, n, width, dtype):
    check(gs, *some(groups * beams, n, dtype, groups * 100 + n), beams, width)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("n", [50, 4096, 50_000, 200_001])
@pytest.mark.parametrize("width", [1, 8, 130])
def test_equal_scores(gs, n, width, dtype):
    """All equal; few distinct values; equal rows: the lowest walk, and the lowest node."""
    beams = 4
    logp = torch.tensor([-1.0, -1.0, -2.0, -1.0] * 2, device=DEV)
    check(gs, torch.zeros(8, n, dtype=TORCH[dtype], device=DEV), logp, beams, width)
    gen = torch.Generator().manual_seed(n)
    one = torch.randint(-3, 3, (1, n), generator=gen).to(TORCH[dtype]).to(DEV)
    check(gs, one.repeat(8, 1), logp, beams, width)
    check(gs, torch.randint(-2, 2, (8, n), generator=gen).to(TORCH[dtype]).to(DEV), logp, beams, width)
    zeros = torch.zeros(8, n, dtype=TORCH[dtype])
    zeros[:, ::3] = -0.0
    check(gs, zeros.to(DEV), logp, beams, width)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("n", [3, 1000, 33_000])
def test_masks_ends_and_missing_walks(gs, n, dtype):
    beams, width = 6, 20
    z, logp = some(4 * beams, n, dtype, n, masked=0.4)
    z[1], z[8, 1:], z[9, :-1], z[13] = -INF, -INF, -INF, torch.nan
    z[2, ::2] = torch.nan
    logp[3], logp[4], logp[5] = -INF, torch.nan, 0.0
    ended = torch.zeros(4 * beams, dtype=torch.bool, device=DEV)
    ended[[0, 4, 7, 14]] = True
    z[7] = torch.nan                                   # not looked at
    logp[3 * beams:] = -INF                            # a group without walks
    ended[3 * beams + 1] = True
    got = check(gs, z, logp, beams, width, ended)
    assert int((got[0][3] != -1).sum()) == 0 and bool((got[2][3] == -INF).all())
    check(gs, z, logp, beams, width, ended.to(torch.uint8) * 255)
    check(gs, z, logp, beams, width)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("n", [40, 20_000])
def test_infinities_and_largest_values(gs, n, dtype):
    z, logp = some(8, n, dtype, 3)
    z[0, 5] = INF
    z[1, ::7] = INF
    z[2] = INF
    z[3] = torch.finfo(TORCH[dtype]).max
    z[4] = torch.finfo(TORCH[dtype]).min
    z[5, n // 2] = torch.finfo(TORCH[dtype]).max
    z[6] *= 1e-30 if dtype != "f16" else 1e-5
    check(gs, z, logp, 4, 9)
    check(gs, z, torch.zeros(8, device=DEV), 8, 30)


def test_equal_p_of_different_scores(gs):
    """Scores so small that their differences vanish in p: still by score inside a row."""
    z = torch.tensor([[1e-30, 3e-30, 2e-30, 0.0], [0.0, 0.0, 0.0, 1e-38]], device=DEV)
    parents, nodes, _ = gs.gs_beam_select(z, torch.zeros(2, device=DEV), 2, 8)
    assert parents.tolist() == [[0, 0, 0, 0, 1, 1, 1, 1]] and nodes.tolist() == [[1, 2, 0, 3, 3, 0, 1, 2]]


@pytest.mark.parametrize("dtype", list(TORCH))
def test_far_walks(gs, dtype):
    """One walk far ahead of all others: everything comes from its row; and sums of walks far below."""
    z, logp = some(12, 6000, dtype, 5)
    logp[3] = 1000.0
    logp[7] = -1e30
    check(gs, z, logp, 12, 100)
    check(gs, z, logp * 1e3, 4, 100)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_at_odd_addresses(gs, dtype):
    n, rows = 4097, 6
    room = torch.full((rows * n + 9,), 60.0, dtype=TORCH[dtype], device=DEV)
    z = room[1:1 + rows * n].view(rows, n)
    z.copy_(some(rows, n, dtype, 4)[0])
    check(gs, z, torch.zeros(rows, device=DEV), 3, 7)


def test_ascending_and_descending_rows(gs):
    n = 100_000
    up = torch.linspace(-5, 5, n, device=DEV)
    check(gs, torch.stack([up, up.flip(0), up.roll(n // 2), up.roll(100)]), torch.tensor([0.0, -1e-3, -2e-3, -3e-3], device=DEV), 4, 64)
    step = torch.zeros(2, n, device=DEV)               # 200 good nodes, all in one lane's places or side by side
    step[0, 1024 * torch.arange(90) + 5] = torch.arange(90, dtype=torch.float32, device=DEV) / 10
    step[1, 300:500] = 3.0
    check(gs, step, torch.zeros(2, device=DEV), 2, 250)


def test_many_scores(gs):
    """More than 2^31 scores; the last row counts."""
    n, rows = 70_000_001, 31
    z = torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV)
    z[-1, -1], z[0, 3], z[-1, 40_000_000] = 40.0, 39.0, 38.0
    parents, nodes, p = gs.gs_beam_select(z, torch.zeros(rows, device=DEV), rows, 3)
    # log exp(39) / (exp(39) + n - 1) is about 0; log exp(40) / (exp(40) + exp(38) + n - 2) about -0.127
    assert parents.tolist() == [[0, 30, 30]] and nodes.tolist() == [[3, n - 1, 40_000_000]]
    two = math.log(math.exp(40) + math.exp(38) + n - 2)
    want = [39 - math.log(math.exp(39) + n - 1), 40 - two, 38 - two]
    assert np.allclose(p.cpu().numpy()[0], want, rtol=2.0 ** -23, atol=1e-11)   # differences of numbers of 39: 2^-47 each


def test_captured_and_replayed(gs):
    beams, n, width = 5, 30_001, 6
    z, logp = some(3 * beams, n, "bf16", 1)
    ws = torch.empty(gs.gs_beam_select_workspace_bytes(3, beams, n, width, gs.GS_BF16), dtype=torch.uint8, device=DEV)
    outs = gs.gs_beam_select(z, logp, beams, width, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gs.gs_beam_select(z, logp, beams, width, parents_out=outs[0], nodes_out=outs[1], logp_out=outs[2], ws=ws)
    for seed in range(4):
        a, b = some(3 * beams, n, "bf16", seed)
        z.copy_(a)
        logp.copy_(b)
        [x.fill_(9) for x in outs]
        graph.replay()
        torch.cuda.synchronize()
        first = [x.clone() for x in outs]
        ws.fill_(255)
        assert all(torch.equal(x, y) for x, y in zip(first, check(gs, z, logp, beams, width)))


# ---- what is kept for each walk -------------------------------------------------

def moved(state, parents, beams, out):
    groups, width = parents.shape
    want = out.clone()
    for g in range(groups):
        for k in range(width):
            b = int(parents[g, k])
            if 0 <= b < beams:
                want[g * width + k] = state[g * beams + b]
    return want


def state_of(rows, shape, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(0, 256, (rows, *shape), generator=gen, dtype=torch.int32).to(dtype).to(DEV)


SHAPES = [((1,), torch.uint8), ((3,), torch.uint8), ((17,), torch.int16), ((80,), torch.int32), ((1,), torch.float32), ((128,), torch.float32), ((5, 7), torch.float64),
          ((1000,), torch.bfloat16), ((4099,), torch.uint8), ((3, 5000), torch.float32), ((16_384,), torch.float32), ((0,), torch.float32), ((), torch.int64)]


@pytest.mark.parametrize("groups,beams,width", [(1, 1, 1), (1, 4, 4), (3, 4, 6), (7, 8, 3), (2, 1, 9), (1, 256, 256), (2, 100, 65), (130, 3, 3)])
def test_reorder_to_others(gs, groups, beams, width):
    gen = torch.Generator().manual_seed(groups + beams)
    parents = torch.randint(-1, beams, (groups, width), generator=gen, dtype=torch.int32)
    parents[0, 0] = beams if beams > 1 else 0
    states = [state_of(groups * beams, shape, t, i) for i, (shape, t) in enumerate(SHAPES)]
    outs = [state_of(groups * width, shape, t, 100 + i) for i, (shape, t) in enumerate(SHAPES)]
    before = [x.clone() for x in states]
    want = [moved(x, parents, beams, o) for x, o in zip(states, outs)]
    gs.gs_beam_reorder(states, parents.to(DEV), beams, outs=outs)
    assert all(torch.equal(x, y) for x, y in zip(outs, want))
    assert all(torch.equal(x, y) for x, y in zip(states, before))


@pytest.mark.parametrize("groups,beams", [(1, 1), (1, 4), (5, 8), (2, 256), (3, 65), (130, 3), (300, 2)])
def test_reorder_in_place(gs, groups, beams):
    gen = torch.Generator().manual_seed(groups + beams)
    for kind in range(4):
        if kind == 0:
            parents = torch.randint(-1, beams + 1, (groups, beams), generator=gen, dtype=torch.int32)
        elif kind == 1:
            parents = torch.arange(beams, dtype=torch.int32).flip(0).repeat(groups, 1)
        elif kind == 2:
            parents = torch.zeros(groups, beams, dtype=torch.int32) + (beams - 1)
        else:
            parents = torch.arange(beams, dtype=torch.int32).roll(1).repeat(groups, 1)
        states = [state_of(groups * beams, shape, t, i) for i, (shape, t) in enumerate(SHAPES)]
        want = [moved(x, parents, beams, x) for x in states]
        gs.gs_beam_reorder(states, parents.to(DEV), beams)
        assert all(torch.equal(x, y) for x, y in zip(states, want))


@pytest.mark.parametrize("length", [1, 2, 3, 4, 5, 80, 1001])
@pytest.mark.parametrize("in_place", [True, False])
def test_reorder_appends(gs, length, in_place):
    groups, beams, width = 9, 5, 5 if in_place else 7
    gen = torch.Generator().manual_seed(length)
    for column in sorted({0, length // 2, length - 1}):
        walks = torch.randint(0, 1000, (groups * beams, length), generator=gen, dtype=torch.int32).to(DEV)
        rows = torch.randn(groups * beams, 33, generator=gen).to(DEV)
        parents = torch.randint(-1, beams, (groups, width), generator=gen, dtype=torch.int32)
        parents[0] = torch.arange(width) % beams
        nodes = torch.randint(-1, 1000, (groups, width), generator=gen, dtype=torch.int32)
        outs = None if in_place else [torch.full((groups * width, length), 5, dtype=torch.int32, device=DEV), torch.zeros(groups * width, 33, device=DEV)]
        want = [moved(x, parents, beams, x if in_place else o) for x, o in zip((walks, rows), outs or (walks, rows))]
        there = (parents >= 0).reshape(-1).to(DEV)
        want[0][there, column] = nodes.reshape(-1).to(DEV)[there]
        gs.gs_beam_reorder([walks, rows], parents.to(DEV), beams, outs=outs, nodes=nodes.to(DEV), columns=[column, None])
        got = [walks, rows] if in_place else outs
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_reorder_some_in_place_and_many(gs):
    """More states than one launch takes, every other one in place, at odd addresses."""
    groups, beams = 6, 4
    parents = torch.randint(0, beams, (groups, beams), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    states, outs, want, room = [], [], [], []
    for i in range(150):
        r = state_of(1, (groups * beams * (i + 1) + 3,), torch.uint8, i)[0]
        room.append(r)
        states.append(r[i % 3:i % 3 + groups * beams * (i + 1)].view(groups * beams, i + 1))
        outs.append(None if i % 2 else torch.zeros_like(states[-1]))
        want.append(moved(states[-1], parents, beams, states[-1]))
    gs.gs_beam_reorder(states, parents.to(DEV), beams, outs=outs)
    assert all(torch.equal(x if o is None else o, w) for x, o, w in zip(states, outs, want))


def test_reorder_large_rows(gs):
    """A state of more than 2^32 bytes, to another buffer and in place."""
    groups, beams, columns = 2, 3, 90_000_000
    state = torch.zeros(groups * beams, columns, dtype=torch.int64, device=DEV)
    mark = torch.arange(groups * beams, device=DEV) + 1
    for at in (0, 44_739_243, columns - 1):
        state[:, at] = mark
    parents = torch.tensor([[2, 0, 2], [1, 1, 0]], dtype=torch.int32, device=DEV)
    want = torch.tensor([3, 1, 3, 5, 5, 4], device=DEV)
    out = torch.full_like(state, 7)
    gs.gs_beam_reorder([state], parents, beams, outs=[out])
    gs.gs_beam_reorder([state], parents, beams)
    for x in (out, state):
        assert all(torch.equal(x[:, at], want) for at in (0, 44_739_243, columns - 1)) and int((x != 0).sum()) == 18


def test_a_search(gs):
    """Quantised rows, scores, selection and reordering together: eight steps of three searches, each against plain steps."""
    nodes, dim, groups, beams, length = 2000, 72, 3, 4, 9
    gen = torch.Generator().manual_seed(11)
    w_in, w_out = (torch.randn(nodes, dim, generator=gen).bfloat16().to(DEV) for _ in range(2))
    t_in, t_out = gs.gs_quantize_rows(w_in), gs.gs_quantize_rows(w_out)
    bias = torch.zeros(nodes, device=DEV)
    bias[torch.rand(nodes, generator=gen).to(DEV) < 0.2] = -INF
    starts = torch.tensor([5, 77, 1999], dtype=torch.int32, device=DEV)
    stop = 3                                             # nodes below this one end a walk
    walks = torch.full((groups * beams, length), -1, dtype=torch.int32, device=DEV)
    walks[:, 0] = starts.repeat_interleave(beams)
    rows = gs.gs_get_rows(w_in, walks[:, 0].contiguous())
    logp = torch.full((groups, beams), -INF, device=DEV)
    logp[:, 0] = 0.0
    ended = torch.zeros(groups * beams, dtype=torch.bool, device=DEV)
    plain = walks.cpu().clone()
    for t in range(1, length):
        last = walks[:, t - 1].clamp(min=0).contiguous()
        z = gs.gs_scores_q8(t_in, t_out, last, bias=bias, scale=0.2, dtype=torch.bfloat16)
        z[:, stop:] -= 0.5 * (t == 3)
        parents, picked, new = check(gs, z, logp.reshape(-1).contiguous(), beams, beams, ended)
        gs.gs_beam_reorder([walks, rows], parents, beams, nodes=picked, columns=[t, None])
        plain = moved(plain, parents.cpu(), beams, plain)
        plain[:, t] = torch.where(parents.cpu().reshape(-1) >= 0, picked.cpu().reshape(-1), plain[:, t])
        assert torch.equal(walks.cpu(), plain)
        ended = ended.view(groups, beams).gather(1, parents.long().clamp(min=0)).reshape(-1) | (picked.reshape(-1) < stop)
        logp = new
    assert torch.equal(rows, gs.gs_get_rows(w_in, walks[:, 0].contiguous()))
    assert bool((walks[:, 0].view(groups, beams) == starts[:, None]).all()) and bool((logp[:, :-1] >= logp[:, 1:]).all())


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("n", [1, 63, 64, 1000, 2049, 4096])
@pytest.mark.parametrize("width", [1, 20, 32])
def test_many_short_rows(gs, n, width, dtype):
    """Rows that a wave each takes: all different, few values, all equal, rising; walks that ended or are none in between."""
    groups, beams = 43, 6
    rows = groups * beams
    z, logp = some(rows, n, dtype, n + width)
    gen = torch.Generator().manual_seed(n)
    z[::4] = torch.randint(-2, 2, (z[::4].shape[0], n), generator=gen).to(TORCH[dtype]).to(DEV)
    z[1::8] = 0.5
    z[5::8] = torch.linspace(-3, 3, n).to(TORCH[dtype]).to(DEV)
    z[7::16] = torch.nan
    z[9::32, n // 2] = INF
    logp[::11], logp[3::17] = -INF, -1.0
    ended = (torch.rand(rows, generator=gen) < 0.1).to(DEV)
    check(gs, z, logp, beams, width, ended)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("groups,beams,n,width", [(1, 256, 20, 256), (2, 256, 9000, 40), (3, 130, 2, 200), (1, 64, 40_000, 250)])
def test_more_equal_candidates_than_a_list_takes(gs, groups, beams, n, width, dtype):
    logp = torch.full((groups * beams,), -3.0, device=DEV)
    logp[beams // 2] = -4.0
    check(gs, torch.zeros(groups * beams, n, dtype=TORCH[dtype], device=DEV), logp, beams, width)
    step = torch.zeros(groups * beams, n)
    step[:, 1::2] = 0.25
    check(gs, step.to(TORCH[dtype]).to(DEV), logp, beams, width)


@pytest.mark.parametrize("n", [10, 20_000])
def test_certain_walks(gs, n):
    """log-probabilities of +infinity, and above 0: nothing but an order."""
    z, logp = some(10, n, "f32", 2)
    logp[3], logp[7], logp[8] = INF, 5.0, 5.0
    parents, nodes, p = gs.gs_beam_select(z, logp, 5, 8)
    best = torch.sort(z[3], descending=True, stable=True)[1][:8].int()
    count = min(8, int((z[3] > -INF).sum()))
    assert parents[0, :count].tolist() == [3] * count and bool((p[0, :count] == INF).all()) and torch.equal(nodes[0, :count], best[:count])
    assert bool((p[1] <= 5).all()) and set(parents[1].tolist()) <= {2, 3}


def test_log_probabilities_in_place(gs):
    for groups, beams, n in ((3, 5, 40_000), (70, 8, 900)):
        z, logp = some(groups * beams, n, "bf16", n)
        want = check(gs, z, logp, beams, beams)
        got = gs.gs_beam_select(z, logp, beams, beams, logp_out=logp.view(groups, beams))
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(logp.view(groups, beams), want[2])


def test_two_graphs_of_one_workspace_and_another_stream(gs):
    shapes = [(3, 5, 30_001, 6), (2, 8, 9000, 8)]
    ws = torch.empty(max(gs.gs_beam_select_workspace_bytes(g, b, n, w, gs.GS_F32) for g, b, n, w in shapes), dtype=torch.uint8, device=DEV)
    work, graphs = [], []
    stream = torch.cuda.Stream()
    for g, b, n, w in shapes:
        z, logp = some(g * b, n, "f32", n)
        state = torch.arange(g * b * 7, dtype=torch.int32, device=DEV).view(g * b, 7)
        out = torch.zeros(g * w, 7, dtype=torch.int32, device=DEV)
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            outs = gs.gs_beam_select(z, logp, b, w, ws=ws)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            gs.gs_beam_select(z, logp, b, w, parents_out=outs[0], nodes_out=outs[1], logp_out=outs[2], ws=ws)
            gs.gs_beam_reorder([state], outs[0], b, outs=[out], nodes=outs[1], columns=[6])
        work.append((z, logp, b, w, state, outs, out))
        graphs.append(graph)
    for turn in range(3):
        for z, logp, *_ in work:
            z.copy_(z.roll(turn + 1, 1))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for z, logp, b, w, state, outs, out in work:
            want = check(gs, z, logp, b, w)
            assert all(torch.equal(x, y) for x, y in zip(outs, want))
            rows = moved(state.cpu(), want[0].cpu(), b, out.cpu())
            rows[:, 6] = want[1].reshape(-1).cpu()
            assert torch.equal(out.cpu(), rows)
