"""gs_clip_grads against the definition in 64 bits: the norm to 1e-14 relative (a sum of fp64 squares, each rounded once, in
blocks: some hundred roundings of 2^-53), a scaled element within one rounding to its format of x times a factor that is
itself rounded to fp32 (2^-24), and the product in fp32 (2^-24)."""
import math

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


def tensors(sizes, fmts, seed=0, shift=0):
    """Views at offsets of `shift` elements plus what the sizes leave: every alignment occurs."""
    g = torch.Generator().manual_seed(seed)
    flat = {f: (0.1 * torch.randn(sum(sizes) + shift + 8, generator=g)).to(DTYPES[f]).to(DEV) for f in set(fmts)}
    out, at = [], shift
    for i, s in enumerate(sizes):
        out.append(flat[fmts[i % len(fmts)]][at:at + s])
        at += s
    return out


def norm_of(ts):
    return math.sqrt(sum(float(t.cpu().double().square().sum()) for t in ts))


def check_scaled(got, was, factor):
    for g, w in zip(got, was):
        want = w.cpu().double() * factor
        u = torch.finfo(g.dtype).eps / 2
        least = 2.0 ** -25 if g.dtype == torch.float16 else 0.0
        assert torch.all((g.cpu().double() - want).abs() <= (u + 2 * 2.0 ** -24) * want.abs() + least)


CASES = [[1], [3], [2048 * 4], [2048 * 8 + 1], [5, 0, 7, 1, 1], [100_003, 17, 1, 65_536, 8191], [3] * 300 + [40_000], [1] * 112, [1] * 113, [0, 0]]


@pytest.mark.parametrize("sizes", CASES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("fmts", [("f32",), ("bf16",), ("f16",), ("f32", "bf16", "f16")], ids="-".join)
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_norm_and_clipping(gs, sizes, fmts, shift):
    grads = tensors(sizes, fmts, shift=shift)
    was = [t.clone() for t in grads]
    norm = norm_of(grads)
    got = gs.gs_clip_grads(grads, math.inf)
    assert got.dtype == torch.float64 and abs(got.item() - norm) <= 1e-14 * norm
    assert all(torch.equal(a, b) for a, b in zip(grads, was))
    assert gs.gs_clip_grads(grads, 1.01 * norm + 1).item() == got.item()           # not reached: nothing is written
    assert all(torch.equal(a, b) for a, b in zip(grads, was))
    outs = [torch.full_like(t, 7.0) for t in grads]
    limit = 0.3 * norm
    assert gs.gs_clip_grads(gs.GradList(grads, outs), limit).item() == got.item()
    assert all(torch.equal(a, b) for a, b in zip(grads, was))
    check_scaled(outs, was, 0.3 if norm else 1.0)
    assert gs.gs_clip_grads(grads, limit).item() == got.item()
    assert all(torch.equal(a, b) for a, b in zip(grads, outs))


def test_nothing_around_the_tensors_is_touched(gs):
    whole = torch.ones(1000, device=DEV)
    grads = [whole[3:9], whole[10:500], whole[777:778]]
    gs.gs_clip_grads(grads, 0.0)
    keep = torch.ones(1000, dtype=torch.bool)
    keep[3:9] = keep[10:500] = keep[777:778] = False
    assert torch.all(whole.cpu()[keep] == 1) and torch.all(whole.cpu()[~keep] == 0)


def test_outputs_at_another_alignment_and_partly_in_place(gs):
    grads = tensors([30_001, 7, 9000], ("bf16",), shift=1)
    was = [t.clone() for t in grads]
    room = torch.zeros(40_000, dtype=torch.bfloat16, device=DEV)
    outs = [room[4:30_005], None, room[30_008:39_008]]
    norm = norm_of(grads)
    gs.gs_clip_grads(gs.GradList(grads, outs), norm * 2)
    assert torch.equal(outs[0], was[0]) and torch.equal(grads[1], was[1]) and torch.equal(outs[2], was[2])
    gs.gs_clip_grads(gs.GradList(grads, outs), norm / 2)
    check_scaled([outs[0], grads[1], outs[2]], was, 0.5)
    assert torch.equal(grads[0], was[0]) and torch.equal(grads[2], was[2])


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
def test_a_norm_that_is_no_number_scales_nothing(gs, bad, fmt):
    grads = tensors([5000, 3], (fmt,))
    grads[0][4321] = bad
    was = [t.clone() for t in grads]
    outs = [torch.zeros_like(t) for t in grads]
    norm = gs.gs_clip_grads(gs.GradList(grads, outs), 1.0).item()
    gs.gs_clip_grads(grads, 1.0)
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    bits = torch.int32 if fmt == "f32" else torch.int16
    assert all(torch.equal(a.view(bits), b.view(bits)) and torch.equal(c.view(bits), b.view(bits)) for a, b, c in zip(grads, was, outs))


def test_squares_beyond_fp32(gs):
    for x in (1e30, 1e-30):
        grads = [torch.full((4096,), x, device=DEV)]
        got = gs.gs_clip_grads(grads, x).item()
        assert abs(got - 64 * float(torch.tensor(x))) <= 1e-14 * got
        check_scaled(grads, [torch.full((4096,), x)], x / got)


def test_refusals(gs):
    t = torch.ones(8, device=DEV)
    for limit in (-1.0, math.nan):
        with pytest.raises(gs.GsError) as e:
            gs.gs_clip_grads([t], limit)
        assert e.value.status == gs.GS_EINVAL
    with pytest.raises(TypeError):
        gs.GradList([t], [t.half()])
    with pytest.raises(TypeError):
        gs.GradList([t.double()])
    with pytest.raises(ValueError):
        gs.GradList([torch.ones(4, 4, device=DEV).T])
    with pytest.raises(ValueError):
        gs.GradList([])
    with pytest.raises(gs.GsError) as e:
        gs.gs_clip_grads([t], 1.0, ws=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == gs.GS_EWORKSPACE and torch.all(t == 1)


def test_graph_replays(gs):
    grads, outs = tensors([70_000, 33], ("f32",)), tensors([70_000, 33], ("f32",), seed=1)
    ws = torch.empty(gs.gs_clip_grads_workspace_bytes(2), dtype=torch.uint8, device=DEV)
    norm = torch.zeros(1, dtype=torch.float64, device=DEV)
    plan = gs.GradList(grads, outs)
    gs.gs_clip_grads(plan, 2.0, norm_out=norm, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gs.gs_clip_grads(plan, 2.0, norm_out=norm, ws=ws)
    for k in range(3):
        for g in grads:
            g.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want = norm_of(grads)
        assert abs(norm.item() - want) <= 1e-14 * want
        check_scaled(outs, grads, min(1.0, 2.0 / want))


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_a_factor_below_the_least_float(gs, fmt):
    """A norm of 1e40 clipped to 1e-4: the factor, 1e-44, is a float of three bits; the results, 1e-8, are ordinary."""
    was = torch.full((10_000,), 1e38).to(DTYPES[fmt])
    was[::2] *= -0.37
    grads = [was.to(DEV)]
    norm = norm_of(grads)
    got = gs.gs_clip_grads(grads, 1e-4).item()
    assert abs(got - norm) <= 1e-14 * norm
    check_scaled(grads, [was], 1e-4 / norm)
