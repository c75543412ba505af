"""gs_softmax_loss and gs_scores against the definition in 64 bits.

Bounds (u = half a step of the storage format, v = 2^-24 half a step of fp32, S = scale * sum_d |h_d c_d|, its largest over
the nodes; * are products of fp32 numbers):
  a score z_j carries dz <= (dim + 4) v S + 4 v |z_j|: dim products and sums of the matrix instruction, then scale, bias
  and the change to base 2.  A log-sum moves by no more than the largest dz, exp2 and the sums of a lane add (40 + lanes'
  32-term sums) v: the loss is within 2 dz + 80 v + 4 v |loss|.
  A probability has a relative error of r = 2 dz + 100 v, and u more where it is rounded to 16 bits; sums over n terms in
  fp32 add n v of the sum of absolute values.  Gradients: (r + u16 + n v + 4 v) sum |terms|, then the rounding u |g| to the
  format (for binary16 also half its least step, 2^-25).  A probability below fp32's least normal number, 2^-126, may be 0,
  and so may a result: 2^-126 (1 + f sum |factors|).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
V = 2.0 ** -24


@pytest.fixture(scope="module")
def gs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2407_15452_amd import binding
    binding.lib()
    return binding


def make(n, nodes, dim, fmt, rows=None, seed=0, spread=2.0):
    g = torch.Generator().manual_seed(seed * 7919 + n + 31 * nodes + 1009 * dim)
    sigma = math.sqrt(spread / math.sqrt(dim))
    rows = rows or nodes
    w_in = (sigma * torch.randn(rows, dim, generator=g)).to(DTYPES[fmt])
    w_out = (sigma * torch.randn(nodes, dim, generator=g)).to(DTYPES[fmt])
    c = torch.randint(0, rows, (n,), generator=g, dtype=torch.int32)
    t = torch.randint(0, nodes, (n,), generator=g, dtype=torch.int32)
    return w_in, w_out, c, t


def reference(w_in, w_out, c, t, bias=None, scale=1.0, grad_scale=1.0):
    """Loss, gradients and their bounds in fp64, from the definition (valid ids; context -1: left out)."""
    h, w = w_in.double()[c.long()], w_out.double()
    b = torch.zeros(w.shape[0], dtype=torch.float64) if bias is None else bias.double()
    masked = b == -math.inf
    w = w.masked_fill(masked[:, None], 0.0)
    z = scale * (h @ w.T) + b
    live = (t >= 0) & ~masked[t.clamp(min=0).long()]
    at = t.clamp(min=0).long()[:, None]
    lse = torch.logsumexp(z, 1, keepdim=True)
    loss = (lse - z.gather(1, at))[:, 0]
    p = torch.exp(z - lse)
    p[torch.isinf(lse)[:, 0]] = 0.0
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    coef = (p - hot) * live[:, None]
    size = (p + hot) * live[:, None]
    f = scale * grad_scale
    g_in, g_out = f * coef @ w, f * coef.T @ h
    g_in_abs, g_out_abs = abs(f) * size @ w.abs(), abs(f) * size.T @ h.abs()
    lost = 2.0 ** -126
    g_in_abs, g_out_abs = (g_in_abs, lost * (1 + abs(f) * w.abs().sum(0))), (g_out_abs, lost * (1 + abs(f) * h.abs().sum(0)))
    dim = w.shape[1]
    s_abs = scale * (h.abs() @ w.abs().T)
    finite = z.masked_fill(torch.isinf(z), 0.0)
    dz = ((dim + 4) * V * s_abs + 4 * V * finite.abs()).amax()
    return loss, g_in, g_out, g_in_abs, g_out_abs, float(dz)


def check(gs, w_in, w_out, c, t, fmt, bias=None, scale=1.0, grad_scale=1.0):
    loss, g_in, g_out, g_in_abs, g_out_abs, dz = reference(w_in, w_out, c, t, bias, scale, grad_scale)
    d = [x.to(DEV) for x in (w_in, w_out, c, t)]
    db = None if bias is None else bias.to(DEV)
    got, gi, go = (x.cpu() for x in gs.gs_softmax_loss(*d, bias=db, scale=scale, grad_scale=grad_scale))
    live = t >= 0
    assert torch.all(got[~live] == 0)
    err = (got.double() - loss).abs()[live]
    assert torch.all(err <= 2 * dz + 80 * V + 4 * V * loss.abs()[live]), float(err.max())
    u = torch.finfo(DTYPES[fmt]).eps / 2
    r = 2 * dz + 100 * V + (u if fmt != "f32" else 0.0)
    least = 2.0 ** -25 if fmt == "f16" else 0.0
    for got_g, want, size, terms in ((gi, g_in, g_in_abs, w_out.shape[0]), (go, g_out, g_out_abs, c.numel())):
        assert got_g.dtype == DTYPES[fmt]
        bound = (r + terms * V + 4 * V) * size[0] + size[1]
        bound = bound + u * (want.abs() + bound) + least
        worst = ((got_g.double() - want).abs() - bound).max()
        assert worst <= 0, float(worst)
    alone = gs.gs_softmax_loss(*d, bias=db, scale=scale, want_grad=False)
    assert alone[1] is None and alone[2] is None and torch.equal(alone[0].cpu().isnan(), got.isnan())
    assert torch.all((alone[0].cpu().double() - loss).abs()[live] <= 2 * dz + 80 * V + 4 * V * loss.abs()[live])
    again = gs.gs_softmax_loss(*d, bias=db, scale=scale, grad_scale=grad_scale)
    assert torch.equal(again[0].cpu(), got) and torch.equal(again[1].cpu(), gi) and torch.equal(again[2].cpu(), go)
    return got, gi, go


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(1, 1, 8), (1, 70, 64), (3, 64, 16), (65, 63, 72), (257, 129, 128), (31, 2049, 136),
                                         (300, 1000, 256), (1000, 33, 64), (64, 5000, 40)])
def test_loss_and_gradients(gs, fmt, n, nodes, dim):
    w_in, w_out, c, t = make(n, nodes, dim, fmt)
    if n > 2:
        t[1] = -1
    check(gs, w_in, w_out, c, t, fmt, scale=0.75, grad_scale=1.0 / n)


@pytest.mark.parametrize("fmt,dim", [("f32", 4), ("f32", 68), ("f32", 252), ("bf16", 8), ("f16", 248)])
def test_narrow_and_odd_rows(gs, fmt, dim):
    check(gs, *make(130, 200, dim, fmt, rows=50), fmt)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(5, 37, 24), (140, 700, 128), (33, 4000, 200)])
def test_masked_nodes_and_what_their_rows_hold(gs, fmt, n, nodes, dim):
    """Masked rows of NaN and infinity take no part; offsets do; masked contexts cost infinity and move nothing."""
    w_in, w_out, c, t = make(n, nodes, dim, fmt, seed=3)
    g = torch.Generator().manual_seed(5)
    bias = torch.randn(nodes, generator=g)
    masked = torch.rand(nodes, generator=g) < 0.4
    masked[0], masked[1], masked[-1] = True, False, True
    bias[masked] = -math.inf
    t = torch.where(masked[t.long()], torch.ones_like(t), t)
    clean = check(gs, w_in, w_out, c, t, fmt, bias=bias)
    assert torch.all(clean[2][masked] == 0)
    poisoned = w_out.clone()
    poisoned[masked] = math.nan
    poisoned[0] = math.inf
    d = [x.to(DEV) for x in (w_in, poisoned, c, t)]
    got = gs.gs_softmax_loss(*d, bias=bias.to(DEV))
    for a, b in zip(got, clean):
        assert torch.equal(a.cpu(), b)
    t2 = t.clone()
    t2[2] = 0                                             # a masked context
    got = gs.gs_softmax_loss(d[0], d[1], d[2], t2.to(DEV), bias=bias.to(DEV))
    t2[2] = -1
    left_out = gs.gs_softmax_loss(d[0], d[1], d[2], t2.to(DEV), bias=bias.to(DEV))
    assert float(got[0][2]) == math.inf and torch.all(got[1][2] == 0)
    assert torch.equal(got[2], left_out[2]) and torch.equal(got[1], left_out[1])


def test_everything_masked(gs):
    w_in, w_out, c, t = make(9, 40, 32, "f32")
    bias = torch.full((40,), -math.inf)
    loss, gi, go = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)), bias=bias.to(DEV))
    assert torch.all(loss == math.inf) and torch.all(gi == 0) and torch.all(go == 0)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_ids_that_are_no_rows(gs, fmt):
    w_in, w_out, c, t = make(40, 90, 64, fmt, rows=20)
    c[3], c[4], t[5], t[6], t[7] = 20, -1, 90, -2, -1
    d = [x.to(DEV) for x in (w_in, w_out, c, t)]
    loss, gi, go = gs.gs_softmax_loss(*d)
    bad = [3, 4, 5, 6]
    assert torch.isnan(loss[bad]).all() and float(loss[7]) == 0 and torch.isfinite(loss).sum() == 36
    assert torch.all(gi[bad + [7]] == 0)
    c[3], c[4] = 0, 0
    t[bad] = -1
    same = gs.gs_softmax_loss(d[0], d[1], c.to(DEV), t.to(DEV))
    assert torch.equal(same[2], go) and torch.equal(same[1], gi)


def test_a_row_that_holds_nan_spoils_what_it_touches_alone(gs):
    w_in, w_out, c, t = make(70, 300, 64, "f32")
    c = torch.arange(70, dtype=torch.int32)
    w_in[7] = math.nan
    loss, gi, _ = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)))
    assert torch.isnan(loss).nonzero().flatten().tolist() == [7] and torch.isnan(gi[7]).all()
    assert torch.isfinite(gi[[i for i in range(70) if i != 7]]).all()


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
def test_large_scores_do_not_overflow(gs, fmt):
    """Scores of hundreds: exp of them overflows, exp of their distance to the maximum does not."""
    w_in, w_out, c, t = make(70, 400, 64, fmt, spread=300.0)
    check(gs, w_in, w_out, c, t, fmt, grad_scale=1 / 64)


def test_small_probabilities_count_in_binary16(gs):
    """Equal scores of 60,000 nodes: every probability is 2^-16, the row sums only exist as the sum of all."""
    nodes, dim = 60_000, 8
    w_in, w_out = torch.zeros(4, dim, dtype=torch.float16), torch.ones(nodes, dim, dtype=torch.float16)
    c = t = torch.arange(4, dtype=torch.int32)
    loss, gi, go = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)))
    assert torch.allclose(loss.cpu().double(), torch.full((4,), math.log(nodes), dtype=torch.float64), rtol=4 * V, atol=0)
    assert gi.abs().max() <= (2.0 ** -11 + nodes * V) and torch.all(go == 0)


def test_gradient_against_differences(gs):
    """(L(w + t d) - L(w - t d)) / 2t for each table.  z moves on a line a, so the third derivative of a pair's loss is a third
    central moment of a under p: at most 0.1 (max a - min a)^3.  Differences of two losses carry twice their own error."""
    n, nodes, dim, step = 24, 150, 32, 2.0 ** -5
    w_in, w_out, c, t = make(n, nodes, dim, "f32", rows=n)
    c = torch.arange(n, dtype=torch.int32)
    d = [x.to(DEV) for x in (w_in, w_out, c, t)]
    _, gi, go = gs.gs_softmax_loss(*d)
    loss, *_, dz = reference(w_in, w_out, c, t)
    own = float((2 * dz + 80 * V + 4 * V * loss.abs()).sum())
    g = torch.Generator().manual_seed(1)
    for k, grad in ((0, gi), (1, go)):
        way = torch.randn(d[k].shape, generator=g) * 0.25
        up, down = list(d), list(d)
        up[k], down[k] = (w_in, w_out)[k] + step * way, (w_in, w_out)[k] - step * way
        way = ((up[k].double() - down[k].double()) / (2 * step))            # what was taken, after rounding
        a = way[c.long()] @ w_out.double().T if k == 0 else w_in.double()[c.long()] @ way.T
        third = 0.1 * (a.amax(1) - a.amin(1)).pow(3).sum()
        up[k], down[k] = up[k].to(DEV), down[k].to(DEV)
        high, low = (gs.gs_softmax_loss(*x, want_grad=False)[0].double().sum().item() for x in (up, down))
        slope = float((grad.cpu().double() * way).sum())
        assert abs((high - low) / (2 * step) - slope) <= 1.5 * own / step + step ** 2 / 6 * float(third) + own


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(1, 1, 8), (1, 5000, 128), (33, 777, 72), (200, 65, 256), (64, 300, 64)])
def test_scores(gs, fmt, n, nodes, dim):
    w_in, w_out, c, _ = make(n, nodes, dim, fmt, rows=17)
    bias = torch.randn(nodes, generator=torch.Generator().manual_seed(2))
    for b in (None, bias):
        got = gs.gs_scores(w_in.to(DEV), w_out.to(DEV), c.to(DEV), bias=None if b is None else b.to(DEV), scale=1.5).cpu().double()
        h, w = w_in.double()[c.long()], w_out.double()
        want = 1.5 * (h @ w.T) + (0 if b is None else b.double())
        assert torch.all((got - want).abs() <= (dim + 4) * V * 1.5 * (h.abs() @ w.abs().T) + 4 * V * want.abs() + 2 * V * bias.abs().max())


def test_scores_of_masked_nodes_and_bad_centres(gs):
    w_in, w_out, c, _ = make(40, 200, 64, "bf16", rows=17)
    bias = torch.zeros(200)
    bias[::3] = -math.inf
    w_out[::3] = math.nan
    c[5], c[6] = -1, 17
    got = gs.gs_scores(*(x.to(DEV) for x in (w_in, w_out, c)), bias=bias.to(DEV)).cpu()
    good = [i for i in range(40) if i not in (5, 6)]
    assert torch.all(got[good][:, ::3] == -math.inf) and torch.isfinite(got[good][:, 1::3]).all()
    assert torch.isnan(got[[5, 6]][:, 1::3]).all()


def test_no_pairs(gs):
    w_in, w_out, _, _ = make(4, 50, 64, "bf16")
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    g_out = torch.ones(50, 64, dtype=torch.bfloat16, device=DEV)
    loss, gi, go = gs.gs_softmax_loss(w_in.to(DEV), w_out.to(DEV), none, none, g_out=g_out)
    assert loss.numel() == 0 and gi.shape == (0, 64) and go is g_out and torch.all(go == 0)
    assert gs.gs_scores(w_in.to(DEV), w_out.to(DEV), none).shape == (0, 50)


def test_another_stream_and_graph_replays(gs):
    w_in, w_out, c, t = (x.to(DEV) for x in make(100, 600, 64, "bf16"))
    want = [x.clone() for x in gs.gs_softmax_loss(w_in, w_out, c, t)]
    ws = torch.empty(gs.gs_softmax_loss_workspace_bytes(100, 600, 64, gs.GS_BF16), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(x) for x in want]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda: gs.gs_softmax_loss(w_in, w_out, c, t, loss_out=outs[0], g_in=outs[1], g_out=outs[2], ws=ws)  # noqa: E731
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        for x in outs:
            x.fill_(float(k))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        w_out.add_(0.01)
        want = [x.clone() for x in gs.gs_softmax_loss(w_in, w_out, c, t)]


def test_a_larger_workspace_serves_and_a_smaller_one_does_not(gs):
    w_in, w_out, c, t = (x.to(DEV) for x in make(300, 2000, 128, "f16"))
    need = gs.gs_softmax_loss_workspace_bytes(300, 2000, 128, gs.GS_F16)
    ws = torch.empty(gs.gs_softmax_loss_workspace_bytes(5000, 2000, 128, gs.GS_F16), dtype=torch.uint8, device=DEV)
    a, b = gs.gs_softmax_loss(w_in, w_out, c, t), gs.gs_softmax_loss(w_in, w_out, c, t, ws=ws)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    with pytest.raises(gs.GsError) as e:
        gs.gs_softmax_loss(w_in, w_out, c, t, ws=ws[:need - 256])
    assert e.value.status == gs.GS_EWORKSPACE


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [32, 56, 96, 120, 160, 192, 224, 240])
def test_every_padding_of_a_row(gs, fmt, dim):
    """Rows are padded to a multiple of 32 columns; each has its own layout in LDS."""
    w_in, w_out, c, t = make(150, 333, dim, fmt, rows=60)
    bias = torch.randn(333, generator=torch.Generator().manual_seed(dim))
    bias[::7] = -math.inf
    t = torch.where(t % 7 == 0, t + 1, t).clamp(max=332)
    t[t % 7 == 0] = 1
    check(gs, w_in, w_out, c, t, fmt)
    check(gs, w_in, w_out, c, t, fmt, bias=bias)
    got = gs.gs_scores(w_in.to(DEV), w_out.to(DEV), c.to(DEV)).cpu().double()
    h, w = w_in.double()[c.long()], w_out.double()
    assert torch.all((got - h @ w.T).abs() <= (dim + 4) * V * (h.abs() @ w.abs().T) + 4 * V * (h @ w.T).abs())


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
def test_pairs_without_gradient_spoil_nothing(gs, fmt):
    """Centre rows of NaN and infinity whose pair is left out, or has a masked context, move no row of g_out."""
    w_in, w_out, _, t = make(90, 300, 64, fmt, rows=90)
    c = torch.arange(90, dtype=torch.int32)
    bias = torch.zeros(300)
    bias[11] = -math.inf
    t = torch.where(t == 11, t + 1, t)
    t[5], t[40], t[41] = -1, -1, 11
    d = [x.to(DEV) for x in (w_in, w_out, c, t)]
    clean = gs.gs_softmax_loss(*d, bias=bias.to(DEV))
    w_in[5], w_in[40], w_in[41] = math.nan, math.inf, math.nan
    got = gs.gs_softmax_loss(w_in.to(DEV), *d[1:], bias=bias.to(DEV))
    assert all(torch.equal(a, b) for a, b in zip(got, clean))


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_masked_nodes_stay_masked_beside_rows_that_hold_nan(gs, fmt):
    w_in, w_out, c, t = make(40, 90, 64, fmt, rows=40)
    c = torch.arange(40, dtype=torch.int32)
    bias = torch.zeros(90)
    bias[::3] = -math.inf
    t = torch.where(t % 3 == 0, t + 1, t)
    w_in[7], w_in[8, 3], c[9] = math.nan, math.inf, 40
    d = [x.to(DEV) for x in (w_in, w_out, c, t)]
    _, _, go = gs.gs_softmax_loss(*d, bias=bias.to(DEV))
    assert torch.all(go[::3] == 0) and torch.isnan(go[1::3]).any()
    z = gs.gs_scores(*d[:3], bias=bias.to(DEV))
    assert torch.all(z[:, ::3] == -math.inf) and torch.isnan(z[[7, 9]][:, 1::3]).all()


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(1, 900, 64), (70, 300, 64), (300, 2000, 128), (40, 1000, 256)])
def test_pairs_that_are_nearly_certain(gs, fmt, n, nodes, dim):
    """A context that leads by 5 to 60: loss and gradients keep the size of what the other nodes weigh.  1 - p enters unrounded
    (but for 2^-24 of itself), so every bound of the file's head holds with |p - 1| in the place of p + 1, and the loss, the
    logarithm of one plus the others' sum over the context's weight, moves by 1 - p times what the scores do.  binary16: other
    probabilities below its normal numbers, scaled by 2^11 at least under their row's largest (2^14 under 1 for the table),
    are off by half its least step, 2^-25."""
    w_in, w_out, c, t = make(n, nodes, dim, fmt, rows=n, spread=1.0)
    c = torch.arange(n, dtype=torch.int32)
    lead = torch.linspace(5.0, 60.0, n)
    rows = w_out[t.long()].float()
    w_in = (rows * (lead / rows.square().sum(1))[:, None]).to(DTYPES[fmt])
    f = 0.5
    loss, g_in, g_out, *_, dz = reference(w_in, w_out, c, t, grad_scale=f)
    h, w = w_in.double(), w_out.double()
    z = h @ w.T
    at = t.long()[:, None]
    others = torch.softmax(z, 1).scatter(1, at, 0.0)
    miss = others.sum(1)
    apart = z.scatter(1, at, -math.inf)
    loss = torch.log1p((apart - z.gather(1, at)).exp().sum(1))          # not as a difference of large numbers
    hot = torch.zeros_like(others).scatter_(1, at, 1.0)
    coef, size = others - hot * miss[:, None], others + hot * miss[:, None]
    g_in, g_out = f * coef @ w, f * coef.T @ h
    got, gi, go = (x.cpu() for x in gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)), grad_scale=f))
    r = 2 * dz + 100 * V
    assert torch.all((got.double() - loss).abs() <= miss * r + 4 * V * loss + 2.0 ** -126), float((got.double() - loss).abs().max())
    alone = gs.gs_softmax_loss(*(x.to(DEV) for x in (w_in, w_out, c, t)), want_grad=False)[0].cpu()
    assert torch.all((alone.double() - loss).abs() <= miss * r + 4 * V * loss + 2.0 ** -126)
    u = torch.finfo(DTYPES[fmt]).eps / 2
    r += u if fmt != "f32" else 0.0
    least = 2.0 ** -25 if fmt == "f16" else 0.0
    lost = 2.0 ** -126
    low_in = least * 2.0 ** -11 * f * others.amax(1, keepdim=True) * w.abs().sum(0)
    low_out = least * 2.0 ** -14 * f * h.abs().sum(0)
    for have, want, terms, absolute, low in ((gi, g_in, nodes, f * size @ w.abs(), low_in + lost * (1 + w.abs().sum(0))),
                                             (go, g_out, n, f * size.T @ h.abs(), low_out + lost * (1 + h.abs().sum(0)))):
        bound = (r + terms * V + 4 * V) * absolute + low
        bound = bound + u * (want.abs() + bound) + least
        assert torch.all((have.double() - want).abs() <= bound), float(((have.double() - want).abs() - bound).max())


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,nodes,dim", [(1, 700, 256), (8, 129, 200), (9, 300, 160), (40, 1000, 256), (41, 257, 136), (100, 64, 72), (3, 5000, 64)])
def test_masked_scores_in_every_layout(gs, fmt, n, nodes, dim):
    """Long rows come through LDS, short ones do not, few fp32 centres take no matrix instructions: masked nodes of NaN and
    infinity, centres that are no rows, and the last tile's own number of centres in each."""
    w_in, w_out, c, _ = make(n, nodes, dim, fmt, rows=17)
    bias = torch.randn(nodes, generator=torch.Generator().manual_seed(3))
    masked = torch.rand(nodes, generator=torch.Generator().manual_seed(4)) < 0.3
    masked[0], masked[-1] = True, True
    bias[masked] = -math.inf
    w_out[masked] = math.nan
    w_out[0] = math.inf
    bad = torch.zeros(n, dtype=torch.bool)
    if n > 2:
        c[n - 1], c[1] = -5, 17
        bad[n - 1] = bad[1] = True
    got = gs.gs_scores(w_in.to(DEV), w_out.to(DEV), c.to(DEV), bias=bias.to(DEV), scale=0.5).cpu().double()
    assert torch.all(got[:, masked] == -math.inf) and torch.isnan(got[bad][:, ~masked]).all()
    h, w = w_in.double()[c.long()[~bad]], w_out.double()[~masked]
    want = 0.5 * (h @ w.T) + bias.double()[~masked]
    bound = (dim + 4) * V * 0.5 * (h.abs() @ w.abs().T) + 4 * V * want.abs() + 2 * V * bias[~masked].abs().max()
    assert torch.all((got[~bad][:, ~masked] - want).abs() <= bound)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("n,nodes,dim", [(2000, 33, 24), (1500, 1, 72), (4000, 130, 200), (3000, 70, 96)])
def test_many_pairs_on_few_nodes(gs, fmt, n, nodes, dim):
    """The pairs are split into many parts, which lanes of a workgroup join."""
    w_in, w_out, c, t = make(n, nodes, dim, fmt, rows=500)
    t[::5] = -1
    check(gs, w_in, w_out, c, t, fmt, grad_scale=1.0 / n)
