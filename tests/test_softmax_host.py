"""What gs_softmax_loss, gs_scores, gs_sample_scores and gs_clip_grads refuse, and the sizes they ask for: on the host, before
anything is enqueued.  Pointers are made up and never followed."""
import ctypes as C
import math
import os

import pytest
import torch

P = [C.c_void_p(256 * i) for i in range(12)]
BIG = C.c_size_t(1 << 62)
EINVAL, EWORKSPACE, EOVERFLOW = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2407_15452_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    return binding.lib()


def loss(lib, **k):
    a = dict(w_in=P[1], num_in=100, w_out=P[2], nodes=50, dim=64, dtype=0, centers=P[3], contexts=P[4], pairs=8, bias=P[5], scale=1.0,
             loss=P[6], g_in=P[7], g_out=P[8], grad_scale=1.0, ws=P[9], ws_bytes=BIG)
    a.update(k)
    return lib.gs_softmax_loss(a["w_in"], C.c_int64(a["num_in"]), a["w_out"], C.c_int64(a["nodes"]), C.c_int32(a["dim"]), C.c_int32(a["dtype"]),
                               a["centers"], a["contexts"], C.c_int64(a["pairs"]), a["bias"], C.c_float(a["scale"]), a["loss"], a["g_in"],
                               a["g_out"], C.c_float(a["grad_scale"]), a["ws"], a["ws_bytes"], None)


def scores(lib, **k):
    a = dict(w_in=P[1], num_in=100, w_out=P[2], nodes=50, dim=64, dtype=0, centers=P[3], pairs=8, bias=P[5], scale=1.0, out=P[6], ws=P[9], ws_bytes=BIG)
    a.update(k)
    return lib.gs_scores(a["w_in"], C.c_int64(a["num_in"]), a["w_out"], C.c_int64(a["nodes"]), C.c_int32(a["dim"]), C.c_int32(a["dtype"]),
                         a["centers"], C.c_int64(a["pairs"]), a["bias"], C.c_float(a["scale"]), a["out"], a["ws"], a["ws_bytes"], None)


COMMON = [dict(w_in=None), dict(w_out=None), dict(w_in=C.c_void_p(264)), dict(w_out=C.c_void_p(264)), dict(num_in=0), dict(nodes=0),
          dict(nodes=1 << 31), dict(num_in=1 << 31), dict(pairs=-1), dict(pairs=1 << 31), dict(dim=0), dict(dim=-4), dict(dim=66), dict(dim=260),
          dict(dim=68, dtype=1), dict(dim=68, dtype=2), dict(dtype=3), dict(dtype=-1), dict(centers=None), dict(ws=None),
          dict(ws=C.c_void_p(128)), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf)]


@pytest.mark.parametrize("bad", COMMON + [dict(contexts=None), dict(loss=None), dict(g_in=P[1]), dict(g_out=P[2]), dict(g_in=P[2]),
                                          dict(g_out=P[1]), dict(g_in=P[8]), dict(g_in=C.c_void_p(264)), dict(g_out=C.c_void_p(264)),
                                          dict(grad_scale=math.nan), dict(grad_scale=math.inf)], ids=str)
def test_softmax_loss_refuses(lib, bad):
    assert loss(lib, **bad) == EINVAL


@pytest.mark.parametrize("bad", COMMON + [dict(out=None)], ids=str)
def test_scores_refuses(lib, bad):
    assert scores(lib, **bad) == EINVAL


def test_short_workspaces(lib):
    for dtype in (0, 1, 2):
        for pairs, nodes, dim in ((1, 1, 8), (8, 50, 64), (70_000, 10_000, 64), (4096, 1_000_000, 128), (300, 7, 256)):
            q = (C.c_int64(pairs), C.c_int64(nodes), C.c_int32(dim), C.c_int32(dtype))
            for grad, outs in ((1, {}), (1, dict(g_in=None)), (1, dict(g_out=None)), (0, dict(g_in=None, g_out=None))):
                need = lib.gs_softmax_loss_workspace_bytes(*q, C.c_int32(grad))
                assert need > 0 and need % 256 == 0
                assert loss(lib, pairs=pairs, nodes=nodes, dim=dim, dtype=dtype, ws_bytes=C.c_size_t(need - 1), **outs) == EWORKSPACE
            need = lib.gs_scores_workspace_bytes(*q)
            assert scores(lib, pairs=pairs, nodes=nodes, dim=dim, dtype=dtype, ws_bytes=C.c_size_t(need - 1)) == EWORKSPACE


def test_workspace_of_many_pairs_serves_fewer(lib):
    sizes = sorted({1, 2, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 1000, 4095, 4096, 4097, 65_535, 65_536, 65_537, 131_072,
                    131_073, 200_000, 1_000_000})
    for dtype in (0, 1):
        for nodes in (1, 40, 1000, 10_000, 131_073, 1_000_000, 100_000_000):
            for dim in (64, 128, 256):
                for grad in (0, 1):
                    got = [lib.gs_softmax_loss_workspace_bytes(C.c_int64(b), C.c_int64(nodes), C.c_int32(dim), C.c_int32(dtype), C.c_int32(grad)) for b in sizes]
                    assert got == sorted(got) and got[0] > 0
                got = [lib.gs_scores_workspace_bytes(C.c_int64(b), C.c_int64(nodes), C.c_int32(dim), C.c_int32(dtype)) for b in sizes]
                assert got == sorted(got) and got[0] > 0


def test_sizes_that_are_none(lib):
    ask = lambda *q: lib.gs_softmax_loss_workspace_bytes(C.c_int64(q[0]), C.c_int64(q[1]), C.c_int32(q[2]), C.c_int32(q[3]), C.c_int32(1))  # noqa: E731
    assert ask(-1, 10, 64, 0) == ask(5, 0, 64, 0) == ask(5, 10, 65, 0) == ask(5, 10, 264, 1) == ask(5, 10, 64, 7) == 0
    assert lib.gs_sample_scores_workspace_bytes(C.c_int64(-1), C.c_int64(5), C.c_int32(0)) == 0
    assert lib.gs_sample_scores_workspace_bytes(C.c_int64(1), C.c_int64(0), C.c_int32(0)) == 0
    assert lib.gs_clip_grads_workspace_bytes(C.c_int32(-1)) == 0


def test_launches_too_large_for_one(lib):
    """2^24 workgroups of 256 lanes are 2^32 lanes, which no launch takes: refused before anything is enqueued."""
    assert scores(lib, nodes=(1 << 31) - 1, dim=4) == EOVERFLOW
    assert loss(lib, nodes=(1 << 31) - 1, dim=4) == EOVERFLOW
    assert loss(lib, pairs=1 << 26) == EOVERFLOW              # a wave per pair


def sample(lib, **k):
    a = dict(scores=P[1], rows=4, n=100, dtype=0, u=P[2], ids=P[3], probs=P[4], ws=P[5], ws_bytes=BIG)
    a.update(k)
    return lib.gs_sample_scores(a["scores"], C.c_int64(a["rows"]), C.c_int64(a["n"]), C.c_int32(a["dtype"]), a["u"], None, None, None, None,
                                a["ids"], a["probs"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("bad", [dict(scores=None), dict(scores=C.c_void_p(258)), dict(scores=C.c_void_p(257), dtype=1), dict(rows=-1), dict(n=0),
                                 dict(n=1 << 31), dict(dtype=3), dict(u=None), dict(ids=None), dict(ws=None), dict(ws=C.c_void_p(8))], ids=str)
def test_sample_scores_refuses(lib, bad):
    assert sample(lib, **bad) == EINVAL


def test_sample_scores_other_refusals(lib):
    for rows, n in ((1, 1), (4, 100), (64, 1_000_000), (1, (1 << 31) - 1)):
        need = lib.gs_sample_scores_workspace_bytes(C.c_int64(rows), C.c_int64(n), C.c_int32(0))
        assert need >= 256 and sample(lib, rows=rows, n=n, ws_bytes=C.c_size_t(need - 1)) == EWORKSPACE
    assert sample(lib, rows=1 << 22) == EOVERFLOW
    assert sample(lib, rows=0, scores=None, u=None, ids=None) == 0


def clip(lib, items, limit=1.0, norm=P[1], ws=P[2], ws_bytes=BIG):
    from paper_2407_15452_amd.binding import TensorStruct
    array = (TensorStruct * max(1, len(items)))(*[TensorStruct(*i) for i in items])
    return lib.gs_clip_grads(array, C.c_int32(len(items)), C.c_double(limit), norm, ws, ws_bytes, None)


@pytest.mark.parametrize("item", [(None, None, 4, 0), (258, None, 4, 0), (257, None, 4, 1), (256, 1026, 4, 0), (256, None, -1, 0),
                                  (256, None, (1 << 40) + 1, 0), (256, None, 4, 3)], ids=str)
def test_clip_grads_refuses(lib, item):
    assert clip(lib, [(256, None, 4, 0), item]) == EINVAL


def test_clip_grads_other_refusals(lib):
    good = [(256, None, 4, 0)]
    assert clip(lib, good, limit=-0.5) == clip(lib, good, limit=math.nan) == EINVAL
    assert clip(lib, good, norm=None) == clip(lib, good, ws=None) == clip(lib, good, ws=C.c_void_p(16)) == EINVAL
    assert clip(lib, [(256, None, 1 << 40, 0), (256, None, 1, 0)]) == EINVAL
    for n in (1, 112, 113, 1000):
        need = lib.gs_clip_grads_workspace_bytes(C.c_int32(n))
        assert clip(lib, good * n, ws_bytes=C.c_size_t(need - 1)) == EWORKSPACE


def test_binding_refuses_what_the_library_cannot_see():
    """Shapes and types that do not belong together; tensors that are not on the GPU."""
    from paper_2407_15452_amd import binding as gs
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    ids = torch.zeros(3, dtype=torch.int32)
    for w_in, w_out in ((f(4, 8), f(4, 12)), (f(4, 8), f(4, 8).half()), (f(8), f(4, 8)), (f(4, 8).double(), f(4, 8).double())):
        with pytest.raises(TypeError):
            gs.gs_softmax_loss(w_in, w_out, ids, ids)
        with pytest.raises(TypeError):
            gs.gs_scores(w_in, w_out, ids)
    with pytest.raises(ValueError):
        gs.gs_softmax_loss(f(4, 8), f(5, 8), ids, ids, bias=f(4))
    with pytest.raises(ValueError):
        gs.gs_softmax_loss(f(4, 8), f(5, 8), ids, ids[:2])
    with pytest.raises(ValueError):
        gs.gs_softmax_loss(f(4, 8), f(5, 8), ids, ids, g_out=f(4, 8))
    with pytest.raises(ValueError):
        gs.gs_sample_scores(f(3, 5), f(2))
    with pytest.raises(ValueError):
        gs.gs_sample_scores(f(3, 5), f(3), top_p=f(1))
    with pytest.raises(TypeError):
        gs.gs_softmax_loss(f(4, 8), f(5, 8), ids, ids)
    with pytest.raises(TypeError):
        gs.gs_scores(f(4, 8), f(5, 8), ids)
    with pytest.raises(TypeError):
        gs.gs_sample_scores(f(3, 5), f(3))
    with pytest.raises(TypeError):
        gs.GradList([f(4)])
