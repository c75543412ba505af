"""gs_scores_q8 against products in 64 bits of the values that the bytes stand for.

Tolerance: the products of two e4m3 values and two powers of two are exact in fp32, and their sum has one rounding for each
term at most (2^-23 each, if the matrix instruction truncates) of a partial sum that is below S = sum |a_k c_k|; then `scale`
and the bias round once each, and a 16-bit result once more by half a step.  The 8-bit matrix instruction, for 16-bit results, drops
of eight neighbouring products what lies below 2^-13 of the largest: 7 * 2^-13 of it at most, and the largest ones are at most S."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
INF = float("inf")


@pytest.fixture(scope="module")
def gs():
    from paper_2407_15452_amd import binding
    binding.lib()
    return binding


def table(gs, n, dim, seed, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    width = -(-dim // 8) * 8
    x = torch.randn(n, width, generator=gen) * torch.exp(spread * torch.randn(n, 1, generator=gen)) / dim ** 0.25
    x = x[:, :dim] if dim % 4 == 0 else x
    t = gs.gs_quantize_rows(x.contiguous().to(DEV))
    return t


def values(t):
    at = torch.arange(t.dim, device=DEV) // 128
    return t.data.double()[:, :t.dim] * t.scales.double()[:, at]


def check(gs, t_in, t_out, centers, bias=None, scale=1.0, dtype="f32", got=None):
    if got is None:
        got = gs.gs_scores_q8(t_in, t_out, centers, bias=bias, scale=scale, dtype=TORCH[dtype])
    n = t_in.num_nodes
    there = (centers >= 0) & (centers < n)
    h = values(t_in)[centers.long().clamp(0, n - 1)]
    c = values(t_out)
    want = scale * (h @ c.T.contiguous())
    size = scale * (h.abs() @ c.abs().T.contiguous())
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    want[~there] = torch.nan
    if bias is not None:
        want[:, bias == -INF] = -INF
    assert got.dtype == TORCH[dtype] and tuple(got.shape) == tuple(want.shape)
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got == -INF, want == -INF)
    fine = torch.isfinite(want)
    tolerance = ((t_out.dim + 2) * 2.0 ** -23 + (0 if dtype == "f32" else 7 * 2.0 ** -13)) * size + HALF_STEP[dtype] * want.abs() + (2.0 ** -25 if dtype == "f16" else 0.0)
    off = (got - want).abs()
    assert bool((off <= tolerance)[fine].all()), float((off / tolerance)[fine].max())


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("centers,nodes,dim", [
    (1, 1, 4), (1, 1, 8), (1, 31, 16), (2, 33, 64), (1, 1000, 128), (16, 129, 128), (17, 4097, 100), (31, 64, 132), (32, 63, 256), (33, 255, 200),
    (1, 70_001, 64), (4, 10_007, 384), (64, 1000, 512), (65, 257, 640), (100, 3001, 1024), (129, 511, 136), (200, 130, 2056), (255, 1025, 128),
    (256, 256, 256), (257, 513, 260), (300, 300, 8192), (1, 5000, 8192), (777, 1001, 200), (1025, 70, 72), (500, 2049, 1000)])
def test_scores(gs, centers, nodes, dim, dtype):
    t_in, t_out = table(gs, 300, dim, 1), table(gs, nodes, dim, 2)
    ids = torch.randint(0, 300, (centers,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).to(DEV)
    check(gs, t_in, t_out, ids, dtype=dtype, scale=0.5 if dim == 200 else 1.0)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("centers,nodes,dim", [(33, 800_003, 16), (64, 790_001, 128), (600, 172_543, 100), (130, 400_007, 64), (130, 400_064, 64), (700, 30_016, 256)])
def test_many_nodes(gs, centers, nodes, dim, dtype):
    """Long ranges of nodes for each workgroup, in rows that begin inside and on lines of 128 bytes; an output that begins elsewhere."""
    t_in, t_out = table(gs, 300, dim, 1), table(gs, nodes, dim, 2)
    gen = torch.Generator().manual_seed(3)
    ids = torch.randint(0, 300, (centers,), generator=gen, dtype=torch.int32).to(DEV)
    ids[centers // 3] = -1
    bias = torch.randn(nodes, generator=gen).masked_fill(torch.rand(nodes, generator=gen) < 0.1, -INF).to(DEV)
    check(gs, t_in, t_out, ids, bias=bias, dtype=dtype)
    room = torch.full((centers * nodes + 100,), 9.0, dtype=TORCH[dtype], device=DEV)
    out = room[37:37 + centers * nodes].view(centers, nodes)
    gs.gs_scores_q8(t_in, t_out, ids, dtype=TORCH[dtype], out=out)
    assert torch.equal(out.nan_to_num(7.0), gs.gs_scores_q8(t_in, t_out, ids, dtype=TORCH[dtype]).nan_to_num(7.0))
    assert bool((room[:37] == 9).all()) and bool((room[-63:] == 9).all())


@pytest.mark.parametrize("centers", [1, 5, 40, 130, 300])
@pytest.mark.parametrize("dim", [64, 200, 1024])
def test_masks_and_centres_that_are_no_rows(gs, centers, dim):
    nodes = 2003
    t_in, t_out = table(gs, 50, dim, 4), table(gs, nodes, dim, 5)
    gen = torch.Generator().manual_seed(6)
    ids = torch.randint(0, 50, (centers,), generator=gen, dtype=torch.int32).to(DEV)
    ids[centers // 2] = 50
    if centers > 4:
        ids[0], ids[3], ids[-1] = -1, 2 ** 31 - 1, -2 ** 31
    bias = torch.randn(nodes, generator=gen).to(DEV)
    bias[torch.rand(nodes, generator=gen).to(DEV) < 0.3] = -INF
    bias[0], bias[-1] = -INF, -INF
    for dtype in TORCH:
        check(gs, t_in, t_out, ids, bias=bias, dtype=dtype)
    check(gs, t_in, t_out, ids, bias=torch.full_like(bias, -INF))
    check(gs, t_in, t_out, ids, bias=torch.zeros_like(bias), scale=1e-3)


@pytest.mark.parametrize("centers", [1, 40, 300])
@pytest.mark.parametrize("dim", [64, 300, 1024])
def test_nan_stays_in_its_row(gs, centers, dim):
    """A row of infinities or NaN has the scale NaN: its scores are NaN (or masked), the others are untouched."""
    gen = torch.Generator().manual_seed(7)
    x, y = torch.randn(40, dim, generator=gen), torch.randn(301, dim, generator=gen)
    x[7, dim - 1], y[5, 0], y[17], y[300, dim // 2], y[44] = torch.nan, torch.inf, torch.nan, -torch.inf, torch.inf
    t_in, t_out = gs.gs_quantize_rows(x.to(DEV)), gs.gs_quantize_rows(y.to(DEV))
    ids = (torch.arange(centers, dtype=torch.int32) % 40).to(DEV)
    check(gs, t_in, t_out, ids)
    bias = torch.zeros(301, device=DEV)
    bias[17] = -INF
    check(gs, t_in, t_out, ids, bias=bias, dtype="bf16")


@pytest.mark.parametrize("dim", [16, 144, 1040])
def test_what_lies_behind_a_row_is_no_part_of_it(gs, dim):
    """Rows of a copy that is followed by bytes of NaN; rows that end inside a block beside rows that begin there."""
    n = 70
    whole = gs.Table8.empty(n + 8, dim, DEV)
    whole.data.view(torch.uint8).fill_(0x7f)
    whole.scales.view(torch.uint8).fill_(0xff)
    part = gs.Table8(whole.data[:n], whole.scales[:n], dim)
    x = torch.randn(n, dim, generator=torch.Generator().manual_seed(1)).to(DEV)
    gs.gs_quantize_rows(x, out=part)
    for centers in (1, 33, 260):
        ids = (torch.arange(centers, dtype=torch.int32) % n).to(DEV)
        check(gs, part, part, ids)


@pytest.mark.parametrize("dim,power", [(128, 60), (128, -60), (512, 55), (64, -126)])
def test_scales_far_from_one(gs, dim, power):
    gen = torch.Generator().manual_seed(9)
    x = gs.gs_quantize_rows(torch.ldexp(torch.randn(20, dim, generator=gen), torch.tensor(power)).to(DEV))
    y = gs.gs_quantize_rows(torch.ldexp(torch.randn(200, dim, generator=gen), torch.tensor(-power)).to(DEV))
    for centers in (3, 200):
        check(gs, x, y, (torch.arange(centers, dtype=torch.int32) % 20).to(DEV))


def test_no_centres(gs):
    t = table(gs, 10, 64, 1)
    assert tuple(gs.gs_scores_q8(t, t, torch.zeros(0, dtype=torch.int32, device=DEV)).shape) == (0, 10)


@pytest.mark.parametrize("centers,dim", [(1, 128), (7, 1000), (40, 128), (300, 512)])
def test_a_view_of_the_output(gs, centers, dim):
    """An output that begins at an odd element; what surrounds it stays."""
    nodes = 1003
    t_in, t_out = table(gs, 30, dim, 1), table(gs, nodes, dim, 2)
    ids = (torch.arange(centers, dtype=torch.int32) % 30).to(DEV)
    for dtype in TORCH:
        room = torch.full((centers * nodes + 7,), 123.0, dtype=TORCH[dtype], device=DEV)
        out = room[3:3 + centers * nodes].view(centers, nodes)
        got = gs.gs_scores_q8(t_in, t_out, ids, dtype=TORCH[dtype], out=out)
        check(gs, t_in, t_out, ids, dtype=dtype, got=got)
        assert bool((room[:3] == 123).all()) and bool((room[-4:] == 123).all())


@pytest.mark.parametrize("centers,nodes,dim", [(1, 30_000, 128), (48, 3000, 200), (300, 2000, 1024)])
def test_same_bits_captured_and_replayed(gs, centers, nodes, dim):
    t_in, t_out = table(gs, 100, dim, 1), table(gs, nodes, dim, 2)
    ids = torch.randint(0, 100, (centers,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).to(DEV)
    ws = torch.empty(max(256, gs.gs_scores_q8_workspace_bytes(centers, nodes, dim)), dtype=torch.uint8, device=DEV)
    out = torch.empty(centers, nodes, device=DEV)
    gs.gs_scores_q8(t_in, t_out, ids, out=out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gs.gs_scores_q8(t_in, t_out, ids, out=out, ws=ws)
    for seed in range(4):
        ids.copy_(torch.randint(0, 100, (centers,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        again = out.clone()
        ws.fill_(255)
        assert torch.equal(again, gs.gs_scores_q8(t_in, t_out, ids))
    check(gs, t_in, t_out, ids, got=again)


def test_agrees_with_scores_of_the_same_values(gs):
    """The rows' values as an fp32 table, through gs_scores: the same scores but for the order of sums."""
    t_in, t_out = table(gs, 60, 128, 1), table(gs, 900, 128, 2)
    ids = torch.arange(60, dtype=torch.int32, device=DEV)
    wide = gs.gs_scores(values(t_in).float(), values(t_out).float(), ids)
    size = values(t_in).abs() @ values(t_out).abs().T.contiguous()
    assert bool(((gs.gs_scores_q8(t_in, t_out, ids).double() - wide.double()).abs() <= 2 * 130 * 2.0 ** -23 * size).all())


@pytest.mark.parametrize("centers", [1, 200])
def test_tables_beyond_32_bits(gs, centers):
    """A table of more than 2^32 bytes, wide rows; the last ones count."""
    n, dim = 530_000, 8192
    t_out = gs.Table8.empty(n, dim, DEV)
    t_out.data.view(torch.uint8).zero_()
    t_out.scales.view(torch.uint8).fill_(127)
    rows = torch.tensor([0, 262_143, 262_144, 524_287, 524_288, n - 1], device=DEV)
    small = table(gs, 6, dim, 3)
    t_out.data.view(torch.uint8)[rows] = small.data.view(torch.uint8)
    t_out.scales.view(torch.uint8)[rows] = small.scales.view(torch.uint8)
    t_in = table(gs, 9, dim, 4)
    ids = (torch.arange(centers, dtype=torch.int32) % 9).to(DEV)
    got = gs.gs_scores_q8(t_in, t_out, ids)
    check(gs, t_in, small, ids, got=got[:, rows].contiguous())
    got[:, rows] = 0
    assert int((got != 0).sum()) == 0
    far = gs.gs_scores_q8(t_out, small, rows.to(torch.int32))
    check(gs, small, small, torch.arange(6, dtype=torch.int32, device=DEV), got=far)


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("centers,nodes,dim", [(128, 4097, 260), (129, 6200, 384), (300, 5001, 300), (1025, 4100, 640), (513, 2176, 1100)])
def test_tiles_over_groups_of_nodes(gs, centers, nodes, dim, dtype):
    """Several groups of 2048 nodes, the last one ragged; masked nodes and centres that are no row among them."""
    t_in, t_out = table(gs, 400, dim, 5), table(gs, nodes, dim, 6)
    gen = torch.Generator().manual_seed(nodes)
    ids = torch.randint(-1, 401, (centers,), generator=gen, dtype=torch.int32).to(DEV)
    bias = torch.randn(nodes, generator=gen)
    bias[::13] = -INF
    check(gs, t_in, t_out, ids, bias=bias.to(DEV), scale=0.5, dtype=dtype)


def test_on_two_streams_at_once(gs):
    """Calls with workspaces of their own on two streams; each waits for its inputs alone."""
    t_in, t_out = table(gs, 200, 700, 7), table(gs, 9000, 700, 8)
    ids = [torch.randint(0, 200, (n,), generator=torch.Generator().manual_seed(n), dtype=torch.int32).to(DEV) for n in (200, 600)]
    want = [gs.gs_scores_q8(t_in, t_out, i, dtype=torch.bfloat16) for i in ids]
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for turn in range(3):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got[k] = gs.gs_scores_q8(t_in, t_out, ids[k], dtype=torch.bfloat16)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
